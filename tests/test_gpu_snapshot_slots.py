"""GPU: a snapshot built by hand may name any rows for its tokens, those of the sinks among them."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sinks", [1, 3])
def test_sinks_outside_their_rows(sinks):
    import torch

    from paper_2501_04987_amd import binding

    c, d, hkv = 24, 64, 2
    kv = binding.TreeKV(c, hkv, d, kv_heads=hkv, dtype="f32", n_sink=sinks, n_recent=6)
    lay = kv.state_layout()
    g = torch.Generator().manual_seed(3)

    def part(buf, off, dtype, *shape):
        n = torch.Size(shape).numel() * dtype.itemsize
        return buf[off:off + n].view(dtype).view(*shape)

    buf = torch.zeros(lay.bytes, dtype=torch.uint8)
    pos = torch.cat([torch.arange(sinks), torch.arange(c - sinks - 6) * 2 + sinks, torch.arange(94, 100)])
    part(buf, lay.header, torch.int32, hkv, 4)[:] = torch.tensor([c, 100, 5, 0])
    part(buf, lay.positions, torch.int32, hkv, c)[:] = pos
    part(buf, lay.slots, torch.int32, hkv, c)[:] = torch.stack([torch.randperm(c + 1, generator=g)[:c] for _ in range(hkv)])
    part(buf, lay.S, torch.float32, hkv, c)[:] = torch.rand(hkv, c, generator=g)
    part(buf, lay.K, torch.float32, hkv, c, d)[:] = torch.randn(hkv, c, d, generator=g)
    part(buf, lay.V, torch.float32, hkv, c, d)[:] = torch.randn(hkv, c, d, generator=g)
    status = torch.full((hkv,), 9, dtype=torch.int32, device="cuda")
    kv.import_state(buf.cuda(), status)
    out = kv.export_state().cpu()
    assert status.tolist() == [0, 0]
    for off, dtype, shape in ((lay.header, torch.int32, (hkv, 4)), (lay.positions, torch.int32, (hkv, c)),
                              (lay.S, torch.float32, (hkv, c)), (lay.K, torch.float32, (hkv, c, d)),
                              (lay.V, torch.float32, (hkv, c, d))):
        assert torch.equal(part(out, off, dtype, *shape), part(buf, off, dtype, *shape))
