"""GPU: the paged cache at the ends of what its calls accept."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def test_more_columns_than_a_share_can_have(binding):
    """1024 sequences of over 2^20 tokens, whose pages are few that all of them share, and a bound on the chunks that leaves one
    share: a sequence's tokens are a page's rows as often as the page is in its table."""
    import torch

    B, ps, G, d, pages, n = 1024, 256, 32, 64, 6, (1 << 20) + 40
    g = torch.Generator().manual_seed(1)
    kv = binding.PagedKV(pages, ps, G, d, kv_heads=1, batch=B, table_width=n // ps + 1, dtype="f32", tracked=False)
    k, v = [torch.randn(pages, ps, d, generator=g) for _ in "kv"]
    q = torch.randn(B, G, d, generator=g)
    table = torch.randint(0, pages, (B, n // ps + 1), generator=g).int()
    kv.k.copy_(k[:, None])
    kv.v.copy_(v[:, None])
    kv.table.copy_(table)
    kv.lens.fill_(n)
    starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    out, lse = torch.full((B, G, d), 7.0, device="cuda"), torch.full((B, G), 7.0, device="cuda")
    kv.attend(q.cuda(), starts, 256, out, lse)
    out, lse = out.cpu().double(), lse.cpu().double()
    for b in (0, 1, 511, 1022, 1023):
        often = torch.zeros(pages, ps, dtype=torch.float64)
        often += torch.bincount(table[b, :-1].long(), minlength=pages)[:, None]
        often[table[b, -1], :n % ps] += 1
        s = q[b].double() @ k.double().view(-1, d).T * d ** -0.5
        top = s.amax(dim=1, keepdim=True)
        e = often.view(-1) * torch.exp(s - top)
        total = e.sum(dim=1, keepdim=True)
        want, size = e @ v.double().view(-1, d) / total, e @ v.double().abs().view(-1, d) / total
        # a logit as in tests/serve_reference.py; a lane adds up a quarter of its wave's columns, n / 16 of them, each addition off
        # by half a step of the sum, above and below the line
        d_logit = (d + 8) * 2.0 ** -24 * ((q[b].double().abs() @ k.double().abs().view(-1, d).T).amax(dim=1) * d ** -0.5 + s.abs().amax(dim=1))
        eps = 2 * d_logit[:, None] + 2 * (n / 16 + 64) * 2.0 ** -24
        assert bool(((out[b] - want).abs() <= eps * size).all()), float(((out[b] - want).abs() / (eps * size)).max())
        off = (lse[b] - (top + total.log())[:, 0]).abs()
        assert bool((off <= eps[:, 0] + 2.0 ** -22 * lse[b].abs()).all())
