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


def accepted(starts, lens, tokens, longest, cap):
    """The rule of include/treekv.h, sequence by sequence."""
    got, end = [], 0
    for b, n in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        own = 0 <= lo <= hi <= tokens
        if own and hi - lo <= longest and hi - lo <= n <= cap and (hi == lo or lo >= end):
            got.append(b)
        if own and hi > lo:
            end = max(end, hi)
    return got


def held(got, want, room):
    import torch

    off = (got.double().cpu() - want).abs()
    off[got.cpu() == want] = 0.0
    assert bool((off <= room).all()), float((off / room.clamp(min=1e-300)).max())


# Starts that do not ascend from end to end, tokens and the longest chunk; lengths are 40 + 5 b.
ODD = {
    "one far too large": ([0, 2, 100, 6, 8], 8, 2),
    "one negative": ([0, 2, -5, 6, 8], 8, 2),
    "an overlap": ([0, 5, 3, 8, 9], 9, 5),
    "one inside of another": ([0, 9, 2, 4, 12], 12, 9),
    "a row of two": ([0, 4, 3, 3, 8, 10, 9, 12], 12, 5),
    "from the end to the start": ([9, 8, 7, 5, 0], 9, 9),
    "twice the same": ([0, 6, 0, 6, 6], 6, 6),
    "the second half again": (list(range(0, 70, 2)) + list(range(20, 110, 2)), 110, 2),
    "a border of 64 sequences": ([2 * i for i in range(64)] + [2000] + [100 + i for i in range(66)], 200, 2),
    "rows that are nobody's": ([0, 3, 1 << 30, 7, 7, -(1 << 31), 9, 12], 12, 3),
    "chunks of row tiles": ([0, 70, 60, 150, 149, 151, 151, 300], 300, 150),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("name", ODD)
def test_starts_that_do_not_ascend(binding, name, group, dtype):
    """Rows go to the first sequence that has them, the others are refused and left alone, by both calls alike."""
    import torch

    from tests.serve_reference import Paged

    starts, tokens, longest = ODD[name]
    B = len(starts) - 1
    lens = [40 + 5 * b if B < 20 else 20 + b % 7 for b in range(B)]
    if "tiles" in name:
        lens = [n + 200 for n in lens]
    # the reference has the rows of the accepted sequences; the pages of all
    ref = Paged(lens=lens, news=[0] * B, page_size=16, kv_heads=2, group=group, d=64, dtype=dtype, seed=len(name))
    cap = ref.width * 16
    ok = accepted(starts, lens, tokens, longest, cap)
    assert len(ok) < B
    ref.starts, ref.total = torch.tensor(starts, dtype=torch.int32), tokens
    ref.news = [starts[b + 1] - starts[b] if b in ok else 0 for b in range(B)]
    ref.q = torch.randn(tokens, 2 * group, 64, generator=ref.g).to(ref.t)
    kv, dev = ref.on_gpu(binding), ref.starts.cuda()
    status = torch.full((B,), 9, dtype=torch.int32, device="cuda")
    k, v = [torch.randn(tokens, 2, 64, generator=ref.g).to(ref.t) for _ in "kv"]
    positions = torch.randint(0, 1 << 20, (tokens,), generator=ref.g).int()
    kv.append(k.cuda(), v.cuda(), dev, positions.cuda(), status)
    # (append has no `longest`)
    fits = accepted(starts, lens, tokens, tokens, cap)
    assert status.tolist() == [0 if b in fits else binding.TREEKV_EINVAL for b in range(B)]
    assert fits == ok, "the cases are chosen so"
    ref.append(k, v, positions)
    for x in ("k", "v", "weights", "positions"):
        assert torch.equal(getattr(kv, x).cpu(), getattr(ref, x)), x

    mine = torch.zeros(tokens, dtype=torch.bool)
    for b in ok:
        assert not bool(mine[starts[b]:starts[b + 1]].any())
        mine[starts[b]:starts[b + 1]] = True
    for weigh in (False, True):
        want = ref.attend(sequences=ok)
        out, lse = torch.full_like(ref.q, 7.0, device="cuda"), torch.full((tokens, 2 * group), 7.0, device="cuda")
        before = kv.weights.clone()
        status.fill_(9)
        kv.attend(ref.q.cuda(), dev, longest, out, lse, weigh=weigh, status=status)
        assert status.tolist() == [0 if b in ok else binding.TREEKV_EINVAL for b in range(B)]
        held(out.cpu()[mine], want["out"][mine], want["room"][mine])
        held(lse.cpu()[mine], want["lse"][mine], want["lse_room"][mine])
        assert bool((out.cpu()[~mine] == 7.0).all()) and bool((lse.cpu()[~mine] == 7.0).all())
        if not weigh:
            assert torch.equal(kv.weights, before)
            continue
        total = before.double().cpu() + want["gain"]
        held(kv.weights, total, want["gain_room"] + 2.0 ** -23 * total.abs())
        for b in range(B):
            if not ref.news[b]:
                assert torch.equal(kv.weights[b], before[b])


@pytest.mark.parametrize("weigh", [False, True])
def test_starts_that_do_not_ascend_in_every_kernel(binding, weigh):
    """Chunks beside single tokens, weights of many rows in parts, merges of several shares: with two more sequences, one whose
    starts fall and one that begins inside of another's rows, the others come out as without them."""
    import torch

    from tests.serve_reference import Paged

    for lens, news, group, d, dtype in (([900, 300, 40, 1000, 513, 90, 77, 133], [200, 1, 2, 9, 1, 9, 1, 8], 2, 128, "bf16"),
                                        ([700, 400, 300], [600, 100, 300], 3, 64, "bf16"), ([700, 400, 300], [600, 100, 300], 3, 64, "f32"),
                                        ([9000, 400, 3000, 60], [1, 2, 1, 2], 8, 64, "bf16"), ([600, 400, 300, 30], [40, 20, 30, 1], 1, 128, "bf16"),
                                        ([300, 400], [150, 120], 70, 64, "bf16"), ([400] * 70, [1] * 35 + [130] + [1] * 34, 4, 64, "bf16")):
        ref = Paged(lens=lens + [50, 50], news=news + [0, 0], page_size=32, kv_heads=2, group=group, d=d, dtype=dtype, seed=5)
        b, at = len(lens) // 2, ref.starts.tolist()[:-2]
        starts = at + [at[b], at[b + 1]]
        ref.lens[-1] = news[b] + 20
        want, kv = ref.attend(), ref.on_gpu(binding)
        before = kv.weights.clone()
        out, lse = torch.full_like(ref.q, 7.0, device="cuda"), torch.full(ref.q.shape[:2], 7.0, device="cuda")
        status = torch.full((ref.B,), 9, dtype=torch.int32, device="cuda")
        kv.attend(ref.q.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), max(news), out, lse, weigh=weigh, status=status)
        assert status.tolist() == [0] * len(lens) + [binding.TREEKV_EINVAL] * 2
        held(out, want["out"], want["room"])
        held(lse, want["lse"], want["lse_room"])
        if weigh:
            total = before.double().cpu() + want["gain"]
            held(kv.weights, total, want["gain_room"] + 2.0 ** -23 * total.abs())
        else:
            assert torch.equal(kv.weights, before)
        assert torch.equal(kv.weights[-2:], before[-2:])


@pytest.mark.parametrize("weigh", [False, True])
def test_more_sequences_than_shares(binding, weigh):
    """Partial results lie at the borders between shares where sequences outnumber them: some sequences of many shares among others."""
    import torch

    from tests.serve_reference import Paged

    for B, long, hkv, group, d, new, dtype in ((40, (3, 17, 18, 39), 32, 1, 64, 1, "bf16"), (70, (0, 66), 16, 2, 64, 2, "f32"), (20, (1, 2, 19), 16, 7, 128, 40, "bf16"),
                                               (12, (0, 11), 16, 3, 64, 30, "f32"), (9, (4,), 64, 2, 64, 90, "bf16")):
        lens = [3000 if b in long else 40 + b for b in range(B)]
        news = [new if b in long else 1 + b % 2 for b in range(B)]
        ref = Paged(lens=lens, news=news, page_size=32, kv_heads=hkv, group=group, d=d, dtype=dtype, seed=B)
        kv, some = ref.on_gpu(binding), sorted(set(long) | {0, 5})
        out, lse = torch.full_like(ref.q, 7.0, device="cuda"), torch.full(ref.q.shape[:2], 7.0, device="cuda")
        before = kv.weights.clone()
        need = kv.new_attend_scratch(ref.total, new, weigh)
        # scratch ends where it says: what lies behind it stays
        room = torch.full((need.nbytes + 4096,) if need is not None else (4096,), 77, dtype=torch.uint8, device="cuda")
        kv.attend(ref.q.cuda(), ref.starts.cuda(), max(news), out, lse, weigh=weigh, scratch=room[:need.nbytes] if need is not None else None)
        assert bool((room[-4096:] == 77).all())
        ref.hkv, keep = 1, ref.hkv                            # the reference for the first KV head of some sequences
        q, ref.q = ref.q, ref.q[:, :group]
        want = ref.attend(sequences=some)
        ref.hkv, ref.q = keep, q
        for b in some:
            at = slice(int(ref.starts[b]), int(ref.starts[b + 1]))
            held(out[at, :group], want["out"][at], want["room"][at])
            held(lse[at, :group], want["lse"][at], want["lse_room"][at])
            if weigh:
                total = before[b, :1].double().cpu() + want["gain"][b]
                held(kv.weights[b, :1], total, want["gain_room"][b] + 2.0 ** -23 * total.abs())
        # the other heads by their own one-head caches would be the same sums; that none was left out:
        assert not bool((out == 7.0).all(dim=2).any()) and not bool((lse == 7.0).any())
