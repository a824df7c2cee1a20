"""GPU: treekv_qkv_prepare with fp32 storage keeps the bits of its angles."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["pairs", "halves", "planes"])
@pytest.mark.parametrize("d", [64, 128])
def test_sines_and_cosines_are_rounded_once(d, mode):
    """(1, 0) turned is (cos, sin), of near and far positions."""
    import torch

    from paper_2501_04987_amd import binding

    tokens = 4096
    g = torch.Generator().manual_seed(d)
    positions = torch.cat([torch.arange(1024), torch.randint(0, 1 << 20, (tokens - 1024,), generator=g)]).int()
    freq = binding.rope_frequencies(d, 500000.0, device="cpu")
    x = torch.zeros(tokens, 2, d)
    first = torch.arange(d // 2) * 2 if mode == "pairs" else torch.arange(d // 2)
    x[:, :, first] = 1.0
    got = binding.qkv_prepare(x.cuda(), positions=positions.cuda(), inv_freq=freq.cuda(), halves=mode != "pairs",
                              to_planes=mode == "planes")[0].double().cpu()
    at = (first, first + d // 2) if mode == "halves" else (torch.arange(d // 2) * 2, torch.arange(d // 2) * 2 + 1)
    angle = positions.double()[:, None, None] * freq
    for y, want in ((got[..., at[0]], angle.cos()), (got[..., at[1]], angle.sin())):
        # half a step of the result (a product with 1 and a sum with 0 are exact), and of a 64-bit angle: the product, the
        # constant and the product with it on one side, the product on the other, a rounding of 2^-53 each; doubled for the
        # 64-bit functions' own steps
        room = (1 + 2.0 ** -20) * 2.0 ** -24 * want.abs() + 2 * 4 * 2.0 ** -53 * angle + 2.0 ** -51
        off = (y - want).abs()
        assert bool((off <= room).all()), float((off / room).max())
