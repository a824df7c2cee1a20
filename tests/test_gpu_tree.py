"""GPU: treekv_tree_attend and treekv_tree_commit against plain 64-bit forms (tests/speculate_reference.py), against the
chunk and decode paths, and the calls around them: graphs, streams, padded and ragged batches, infinities in hidden places."""
import random

import pytest

from tests import speculate_reference as ref

pytestmark = pytest.mark.gpu
KEEP_LEFT, ACCUMULATED, RERANK = 1, 4, 8


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def tokens(kv, n, seed, scale=1.0):
    """q [B, n, H, d], k and v [B, n, Hkv, d] of the storage type on the GPU."""
    import torch

    c, g = kv.cfg, torch.Generator().manual_seed(seed)
    made = [torch.randn(c.batch, n, h, c.head_dim, generator=g) * s for h, s in ((c.q_heads, 1.5 * scale), (c.kv_heads, 1.0), (c.kv_heads, 1.0))]
    return [x.to(kv.storage_dtype).cuda() for x in made]


def feed(kv, n, seed):
    """n tokens into the cache, in chunks."""
    at = 0
    while at < n:
        L = min(n - at, kv.cfg.max_chunk, 64)
        q, k, v = tokens(kv, L, seed + at)
        out, ret, nret, ev = kv.new_outputs(L)
        kv.prefill_chunk(q, k, v, L, out, ret, nret, ev)
        at += L


def tree(kind, n, rng):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] * n
    if kind == "padded":                                   # absent nodes in the middle and at the end, and children of theirs
        p = [rng.randint(-1, i - 1) if i else -1 for i in range(n)]
        for i in range(n):
            if i % 5 == 3:
                p[i] = rng.choice([-2, -100, i, i + 7, 2 ** 31 - 1, -2 ** 31])
        return p
    return [rng.randint(max(-1, i - 6), i - 1) if i else -1 for i in range(n)]


def make(binding, *, budget=48, batch=2, hkv=2, G=2, d=64, dtype="bf16", flags=0, fed=0, seed=1, **kw):
    kv = binding.TreeKV(budget, hkv * G, d, kv_heads=hkv, batch=batch, dtype=dtype, flags=flags, n_sink=2,
                        n_recent=budget // 3, **kw)
    feed(kv, fed, 1000 * seed)
    return kv


def check_attend(kv, q, k, v, parents, out, lse, every=1, skip=()):
    """Against the plain form, every `every`-th unit and the last."""
    import torch

    c, G = kv.cfg, kv.cfg.q_heads // kv.cfg.kv_heads
    states = ref.state(kv)
    q, k, v = [x.double().cpu() for x in (q, k, v)]
    out, lse = out.double().cpu(), lse.double().cpu()
    for b in range(c.batch):
        for h in range(c.kv_heads):
            if (b * c.kv_heads + h) % every and (b, h) != (c.batch - 1, c.kv_heads - 1):
                continue
            heads = slice(h * G, (h + 1) * G)
            want, want_lse, bound, lse_bound, _ = ref.attend_unit(kv, states[b * c.kv_heads + h], q[b, :, heads], k[b, :, h], v[b, :, h],
                                                                  parents[b])
            for i in skip:
                want_lse[i], want[i] = lse[b, i, heads], out[b, i, heads]
            absent = torch.isinf(want_lse)
            assert torch.equal(torch.isinf(lse[b, :, heads]), absent)
            off = (lse[b, :, heads] - want_lse).abs().masked_fill(absent, 0.0)
            assert bool((off <= lse_bound).all()), (b, h, float(off.max()))
            off = (out[b, :, heads] - want).abs()
            assert bool((off <= bound).all()), (b, h, float((off / (bound + 1e-300)).max()))


SHAPES = [
    # budget, fed, nodes, batch, kv heads, G, head_dim, dtype, flags
    (48, 0, 1, 1, 1, 1, 64, "bf16", 0),                    # an empty cache, one node
    (48, 0, 40, 2, 2, 2, 128, "bf16", 0),
    (48, 1, 7, 2, 1, 1, 64, "f32", 0),
    (48, 17, 33, 2, 2, 4, 64, "bf16", 0),                  # still filling
    (48, 48, 16, 1, 2, 1, 128, "f32", 0),                  # just full
    (48, 133, 32, 2, 2, 8, 128, "bf16", 0),                # evicting
    (300, 450, 256, 1, 1, 1, 64, "bf16", 0),               # the largest tree
    (300, 450, 256, 1, 1, 2, 128, "f32", 0),
    (1000, 1500, 5, 1, 2, 1, 128, "bf16", 0),              # several slices
    (1000, 1500, 5, 1, 2, 4, 64, "f32", 0),
    (200, 333, 31, 40, 4, 1, 64, "bf16", 0),               # many units: one slice
    (100, 150, 20, 16, 8, 4, 128, "bf16", 0),              # many units and rows: 80 rows share tiles
    (100, 70, 33, 16, 8, 4, 64, "bf16", 0),                # two row tiles, still filling
    (300, 450, 256, 5, 8, 1, 128, "bf16", 0),              # the same in slices
    (300, 450, 256, 5, 8, 1, 64, "bf16", 0),
    (100, 150, 12, 8, 8, 4, 128, "bf16", 0),               # 32 rows a workgroup
    (100, 70, 12, 8, 8, 4, 64, "bf16", 0),
    (60, 90, 20, 8, 8, 2, 128, "f32", 0),
    (60, 40, 20, 8, 8, 2, 64, "f32", 0),
    (60, 90, 20, 8, 8, 2, 64, "f32", RERANK),
    (60, 90, 20, 8, 8, 2, 128, "f32", RERANK),
    (48, 0, 3, 1, 1, 2, 64, "bf16", RERANK),
    (48, 30, 21, 2, 2, 2, 128, "bf16", RERANK),
    (48, 133, 40, 2, 2, 4, 64, "bf16", RERANK),
    (300, 700, 13, 1, 2, 8, 128, "bf16", RERANK),
    (48, 133, 40, 6, 2, 4, 64, "bf16", RERANK),            # many units and rows: keys turned for 64 rows
    (300, 700, 13, 7, 2, 8, 128, "bf16", RERANK),
    (200, 90, 70, 30, 1, 2, 128, "bf16", RERANK),          # still filling, three row tiles
    (100, 0, 66, 30, 1, 2, 64, "bf16", RERANK),            # empty
    (300, 450, 33, 2, 1, 1, 64, "f32", RERANK),
    (300, 450, 5, 1, 1, 2, 128, "f32", RERANK),
]


@pytest.mark.parametrize("kind", ["drafted", "chain", "star", "padded"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_attend(binding, shape, kind):
    import torch

    budget, fed, n, batch, hkv, G, d, dtype, flags = shape
    kv = make(binding, budget=budget, batch=batch, hkv=hkv, G=G, d=d, dtype=dtype, flags=flags, fed=fed, seed=n)
    rng = random.Random(n)
    parents = [tree(kind, n, rng) for _ in range(batch)]
    q, k, v = tokens(kv, n, 77)
    before = kv.export_state()
    out, lse, scratch = kv.new_tree_outputs(n)
    out.fill_(7.0), lse.fill_(7.0)
    kv.tree_attend(q, k, v, torch.tensor(parents, dtype=torch.int32, device="cuda"), out, lse, scratch)
    assert torch.equal(before, kv.export_state())          # nothing was changed
    check_attend(kv, q, k, v, parents, out, lse, every=1 if batch * hkv < 20 else 37)
    again = torch.empty_like(out)
    kv.tree_attend(q, k, v, torch.tensor(parents, dtype=torch.int32, device="cuda"), again)    # no lse, scratch of its own
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("flags,batch,G", [(0, 1, 2), (RERANK, 1, 2), (0, 90, 8), (RERANK, 30, 8)])
def test_attend_with_rising_logits(binding, dtype, d, flags, batch, G):
    """Large, ordered logits: every block of columns raises the reference of the sums."""
    import torch

    kv = make(binding, budget=700, batch=batch, hkv=1, G=G, d=d, dtype=dtype, flags=flags)
    q, k, v = tokens(kv, 700, 5)
    direction = torch.randn(d, generator=torch.Generator().manual_seed(1))
    direction = (direction / direction.norm()).cuda()
    k = (k.float() + torch.linspace(-40.0, 40.0, 700, device="cuda")[None, :, None, None] * direction).to(k.dtype)
    for at in range(0, 700, 100):
        out, ret, nret, ev = kv.new_outputs(100)
        kv.prefill_chunk(*[x[:, at:at + 100].contiguous() for x in (q, k, v)], 100, out, ret, nret, ev)
    q, k, v = tokens(kv, 12, 6)
    q = (q.float() + 20.0 * direction).to(q.dtype)
    parents = [tree("drafted", 12, random.Random(3))] * batch
    out, lse, scratch = kv.new_tree_outputs(12)
    kv.tree_attend(q, k, v, torch.tensor(parents, dtype=torch.int32, device="cuda"), out, lse, scratch)
    check_attend(kv, q, k, v, parents, out, lse, every=45)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 128)])
@pytest.mark.parametrize("flags,batch,G", [(0, 1, 1), (RERANK, 1, 1), (0, 90, 8), (RERANK, 30, 8)])
def test_attend_with_keys_of_all_sizes(binding, dtype, d, flags, batch, G):
    """Neighbouring keys and queries differ by powers of two up to 2^60; some are all zeros."""
    import torch

    kv = make(binding, budget=200, batch=batch, hkv=1, G=G, d=d, dtype=dtype, flags=flags)
    n = 12
    q, k, v = tokens(kv, 200, 15)
    power = torch.tensor([2.0 ** ((i * 37) % 61 - 58) for i in range(200)], device="cuda")
    k = (k.float() * power[None, :, None, None]).to(k.dtype)
    k[:, 7::50] = 0
    for at in range(0, 200, 50):
        out, ret, nret, ev = kv.new_outputs(50)
        kv.prefill_chunk(*[x[:, at:at + 50].contiguous() for x in (q, k, v)], 50, out, ret, nret, ev)
    q, k, v = tokens(kv, n, 16)
    q = (q.float() * torch.tensor([2.0 ** (i % 5 - 2) for i in range(n)], device="cuda")[None, :, None, None]).to(q.dtype)
    q[:, 3] = 0
    q[:, 4] *= 2.0 ** 40
    k[:, 1:6] *= 2.0 ** -42
    parents = [tree("chain", n, None)] * batch
    out, lse, scratch = kv.new_tree_outputs(n)
    kv.tree_attend(q, k, v, torch.tensor(parents, dtype=torch.int32, device="cuda"), out, lse, scratch)
    # (the query of 2^40 gives logits of 2^43 to the cached keys near 2^2, whose bound is no bound: it is left out)
    check_attend(kv, q, k, v, parents, out, lse, every=45, skip=(4,))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("batch,G", [(1, 1), (90, 8)])
def test_attend_with_the_lowest_logits(binding, dtype, d, batch, G):
    """Every logit of a query is the same -10^33 or so: the values' mean comes out."""
    import torch

    kv = make(binding, budget=120, batch=batch, hkv=1, G=G, d=d, dtype=dtype)
    q, k, v = tokens(kv, 100, 21)
    q[:], k[:] = 0, 0
    k[..., 0] = 2.0 ** 56
    out, ret, nret, ev = kv.new_outputs(100)
    kv.prefill_chunk(q, k, v, 100, out, ret, nret, ev)
    n = 12
    q2, _, v2 = tokens(kv, n, 22)
    q2[:] = 0
    q2[..., 0] = -(2.0 ** 56)
    parents = torch.tensor([tree("chain", n, None)] * batch, dtype=torch.int32, device="cuda")
    out, lse, scratch = kv.new_tree_outputs(n)
    kv.tree_attend(q2, k[:, :n].contiguous(), v2, parents, out, lse, scratch)
    want_lse = -(2.0 ** 112) * kv.cfg.softmax_scale        # (the log of 112 is nothing beside it)
    assert bool(((lse.double() - want_lse).abs() <= 4 * 2.0 ** -24 * -want_lse).all())
    for i in range(n):
        seen = torch.cat([v[:, :, 0], v2[:, :i + 1, 0]], dim=1).double()
        # sums of 101 + i values, the weights' sum, the quotient: a rounding each
        room = (110 + i) * 2.0 ** -24 * seen.abs().mean(dim=1)
        assert bool(((out[:, i].double() - seen.mean(dim=1)[:, None]).abs() <= room[:, None]).all()), i


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("flags,batch", [(0, 1), (RERANK, 1), (0, 30), (RERANK, 5)])
def test_hidden_infinities_and_nans(binding, dtype, d, flags, batch):
    """A node's rows are not finite: who does not attend it gets the bits it gets without; who does, what arithmetic says."""
    import torch

    kv = make(binding, budget=48, batch=batch, hkv=2, G=4, d=d, dtype=dtype, flags=flags, fed=99)
    n, inf, nan = 40, float("inf"), float("nan")
    parents = [-1, 0, 0, -1, 3, -2, 5] + [rng if rng < 5 else 4 for rng in range(n - 7)]
    par = torch.tensor([parents] * batch, dtype=torch.int32, device="cuda")
    q, k, v = tokens(kv, n, 8)
    clean, lse, scratch = kv.new_tree_outputs(n)
    kv.tree_attend(q, k, v, par, clean, lse, scratch)
    q2, k2, v2 = q.clone(), k.clone(), v.clone()
    v2[0, 2, 0, 3], v2[0, 2, 0, 4], v2[0, 2, 0, 5] = inf, -inf, nan
    v2[0, 39, 1] = nan                                     # the last row, which those behind it repeat
    k2[0, 1, 1] = nan
    k2[0, 5], v2[0, 5], q2[0, 5] = nan, inf, nan           # absent
    k2[0, 6], v2[0, 6] = inf, nan                          # its child
    out, lse2, _ = kv.new_tree_outputs(n)
    kv.tree_attend(q2, k2, v2, par, out, lse2, scratch)
    assert torch.equal(out[1:], clean[1:])
    out, clean = out.cpu()[0], clean.cpu()[0]
    chain = ref.chains(parents)
    for i in range(n):
        for h in range(2):
            heads = slice(h * 4, h * 4 + 4)
            got, want = out[i, heads], clean[i, heads].clone()
            if chain[i] is None:
                assert bool((got == 0).all()) and bool(torch.isinf(lse2[0, i, heads]).all())
                continue
            if h == 1 and 1 in chain[i] or h == 1 and 39 in chain[i]:
                assert bool(torch.isnan(got).all())
                continue
            if h == 0 and 2 in chain[i]:
                assert bool((got[:, 3] == inf).all() and (got[:, 4] == -inf).all() and torch.isnan(got[:, 5]).all())
                got, want = got.clone(), want
                got[:, 3:6] = want[:, 3:6] = 0
            assert torch.equal(got, want), (i, h)
    # two of opposite sign seen together are a NaN
    v3 = v.clone()
    v3[0, 0, 0, 7], v3[0, 1, 0, 7] = inf, -inf
    got = kv.new_tree_outputs(n)[0]
    kv.tree_attend(q, k, v3, par, got, lse2, scratch)
    assert bool(torch.isnan(got[0, 1, :4, 7]).all()) and bool((got[0, 0, :4, 7] == inf).all()) and bool(torch.isfinite(got[0, 3]).all())


def run_commit(kv, q, k, v, parents, paths, longest):
    import torch

    n, c = len(parents[0]), kv.cfg
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse, scratch = kv.new_tree_outputs(n)
    kv.tree_attend(q, k, v, i32(parents), out, lse, scratch)
    retained, nret = kv.new_outputs()[1:3]
    evicted = torch.full((c.batch, c.kv_heads, longest), 77, dtype=torch.int32, device="cuda")
    status = torch.full((c.batch,), 77, dtype=torch.int32, device="cuda")
    kv.tree_commit(q, k, v, i32(parents), lse, i32([p + [-5] * (longest - len(p)) for p in paths]), i32([len(p) for p in paths]),
                   retained, nret, evicted, status)
    return out, retained, nret, evicted, status


COMMITS = [
    # budget, fed, nodes, longest, batch, kv heads, G, head_dim, dtype, flags
    (48, 0, 1, 1, 1, 1, 1, 64, "bf16", 0),
    (48, 0, 40, 40, 2, 2, 2, 64, "bf16", 0),
    (48, 44, 20, 9, 3, 2, 2, 128, "bf16", 0),              # filling and evicting in one commit
    (48, 133, 30, 12, 5, 2, 4, 128, "bf16", 0),
    (48, 48, 70, 70, 2, 1, 1, 64, "f32", 0),               # several sweeps of the tree region, path longer than the cache
    (300, 450, 256, 256, 1, 2, 2, 128, "f32", 0),          # the longest path
    (300, 450, 256, 256, 1, 2, 8, 64, "bf16", 0),
    (1000, 1500, 16, 5, 2, 2, 1, 128, "bf16", 0),
    (48, 133, 30, 6, 2, 2, 2, 64, "bf16", KEEP_LEFT),
    (48, 133, 30, 6, 2, 2, 2, 64, "f32", ACCUMULATED),
    (48, 133, 30, 12, 3, 2, 4, 128, "bf16", RERANK),
    (48, 40, 70, 70, 2, 1, 8, 64, "bf16", RERANK),
    (300, 450, 16, 7, 2, 1, 1, 128, "f32", RERANK),
    (12500, 700, 16, 7, 1, 1, 1, 64, "bf16", 0),           # order arrays beyond on-chip memory
]


@pytest.mark.parametrize("shape", COMMITS, ids=lambda s: "-".join(map(str, s)))
def test_commit(binding, shape):
    import torch

    budget, fed, n, longest, batch, hkv, G, d, dtype, flags = shape
    kv = make(binding, budget=budget, batch=batch, hkv=hkv, G=G, d=d, dtype=dtype, flags=flags, fed=fed, seed=n + 1)
    rng = random.Random(budget + n)
    parents, paths = [], []
    for b in range(batch):
        length = longest if b == 0 else rng.randint(0, longest)
        nodes = sorted(rng.sample(range(n), length))       # the path runs through these, the others go anywhere
        p = [rng.randint(-1, i - 1) if i else -1 for i in range(n)]
        for x, node in enumerate(nodes):
            p[node] = nodes[x - 1] if x else -1
        parents.append(p)
        paths.append(nodes)
    if batch > 3:
        paths[2] = []
    q, k, v = tokens(kv, n, 78)
    before = ref.state(kv)
    _, retained, nret, evicted, status = run_commit(kv, q, k, v, parents, paths, longest)
    after = ref.state(kv)
    assert status.tolist() == [0] * batch
    qd, kd, vd = [x.double().cpu() for x in (q, k, v)]
    for b in range(batch):
        for h in range(hkv):
            u = b * hkv + h
            args = (qd[b, :, h * G:(h + 1) * G], kd[b, :, h], vd[b, :, h], parents[b])
            want, gone, margin = ref.commit_unit(kv, before[u], *args, paths[b])
            assert margin > 1e-5                           # (fp32 scores are off by some 1e-6)
            got = after[u]
            assert evicted[b, h].tolist() == gone + [-1] * (longest - len(gone)), (b, h)
            assert (got["n"], got["t"], got["idx"], got["pos"]) == (want["n"], want["t"], want["idx"], want["pos"]), (b, h)
            assert retained[b, h].tolist() == want["pos"] + [-1] * (budget - want["n"]) and int(nret[b, h]) == want["n"]
            assert torch.equal(got["K"], want["K"]) and torch.equal(got["V"], want["V"])
            # a probability is off by what its logits are (see attend_unit), the sums by a rounding of 2^-24 each and by the
            # accumulators' half step of 2^-41 for every 64 rows
            added = want["S"].clone()
            bound = 0.0
            if paths[b]:
                bound = float(ref.attend_unit(kv, before[u], *args)[3].max())
            room = bound * added + (len(paths[b]) * G + 4) * 2.0 ** -24 * added + (len(paths[b]) * G / 64 + 1) * 2.0 ** -41
            assert bool(((got["S"] - want["S"]).abs() <= room).all()), (b, h, float((got["S"] - want["S"]).abs().max()))


@pytest.mark.parametrize("flags", [0, RERANK])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_commit_of_large_logits(binding, dtype, flags):
    """Logits of some 2^40, where fp32 tells no two probabilities apart: what a column gains is still between 0 and 1 a row."""
    kv = make(binding, batch=1, fed=30, dtype=dtype, flags=flags)
    q, k, v = tokens(kv, 6, 81)
    q *= 2.0 ** 38
    before = ref.state(kv)
    _, _, nret, _, status = run_commit(kv, q, k, v, [[-1, 0, 1, 2, 3, 0]], [[0, 1, 2, 3]], 4)
    assert status.tolist() == [0] and bool((nret == 34).all())
    for old, new in zip(before, ref.state(kv)):
        assert new["pos"][:30] == old["pos"] and bool(new["S"].isfinite().all())
        added = new["S"].clone()
        added[:30] -= old["S"]
        # (4 tokens of 2 heads, and a rounding of a sum below 64)
        assert bool((added >= 0).all()) and bool((added <= 8 + 2.0 ** -18).all()), (float(added.min()), float(added.max()))


@pytest.mark.parametrize("flags", [0, RERANK])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_commit_weighs_with_the_given_lse(binding, dtype, flags):
    """With every lse smaller by 3 each column gains e^3 times as much, past one a row too."""
    import torch

    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    n, parents, path = 6, i32([[-1, 0, 1, 2, 3, 0]]), i32([[0, 1, 2, 3]])
    gains = []
    for less in (0.0, 3.0):
        kv = make(binding, batch=1, fed=30, dtype=dtype, flags=flags)
        q, k, v = tokens(kv, n, 82, scale=3.0)
        before = ref.state(kv)
        out, lse, scratch = kv.new_tree_outputs(n)
        kv.tree_attend(q, k, v, parents, out, lse, scratch)
        kv.tree_commit(q, k, v, parents, lse - less, path, i32([4]), *kv.new_outputs()[1:3])
        gains.append([x["S"] - torch.cat([y["S"], y["S"].new_zeros(4)]) for x, y in zip(ref.state(kv), before)])
    for one, more in zip(*gains):
        assert float(one.max()) > 0.5                      # (so that more is past one)
        # logits and lse below 2^8 in size, in units of log2, are off by 2^-15 at most, the scores (below 2^9) by 2^-15 each time
        assert bool(((more - one * 2.718281828459045 ** 3).abs() <= 2.0 ** -14 * more + 22 * 2.0 ** -15).all())


@pytest.mark.parametrize("flags", [0, RERANK])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rounds_against_chunks_and_steps(binding, flags, dtype):
    """Verify and commit, round after round, sequences accepting different numbers of tokens, against a context of its own for
    each sequence that is fed the same tokens as chunks (one token: a decode step)."""
    import torch

    kw = dict(budget=64, hkv=2, G=2, d=64, dtype=dtype, flags=flags)
    kv = make(binding, batch=3, fed=50, **kw)
    twins = [make(binding, batch=1, **kw) for _ in range(3)]
    for b, twin in enumerate(twins):
        twin.fork(kv, [b], [0])
    rng = random.Random(5)
    for rnd in range(25):
        n = rng.randint(6, 12)
        q, k, v = tokens(kv, n, 500 + rnd)
        parents = [[i - 1 for i in range(6)] + [rng.randint(-1, 5) for _ in range(n - 6)] for _ in range(3)]
        lengths = [rng.randint(0, 6) if rnd % 3 else 1 for _ in range(3)]
        out, retained, nret, evicted, status = run_commit(kv, q, k, v, parents, [list(range(x)) for x in lengths], 6)
        for b, (twin, L) in enumerate(zip(twins, lengths)):
            if L == 0:
                continue
            part = [x[b:b + 1, :L].contiguous() for x in (q, k, v)]
            o, r, nr, ev = twin.new_outputs(None if L == 1 else L)
            if L == 1:
                twin.decode_step(*[x[:, 0].contiguous() for x in part], o, r, nr, ev)
                o, ev = o[:, None], ev[:, :, None]
            else:
                twin.prefill_chunk(*part, L, o, r, nr, ev)
            assert torch.equal(ev[0], evicted[b, :, :L]) and torch.equal(r[0], retained[b]) and torch.equal(nr[0], nret[b])
            # chunks cut P in two bf16 parts (2^-17) and, re-assigned, turned operands too
            assert torch.allclose(out[b, :L], o[0], rtol=0, atol=2e-4 if dtype == "bf16" else 1e-5)
    S = kv.scores()
    for b, twin in enumerate(twins):
        assert torch.allclose(S[b], twin.scores()[0], rtol=1e-4, atol=1e-6)
        assert torch.equal(kv.gather_kv()[0][b], twin.gather_kv()[0][0])


def test_commit_refuses_what_is_no_path(binding):
    import torch

    kv = make(binding, batch=8, fed=100)
    n = 6
    parents = [[-1, 0, 1, 0, -2, 4]] * 8
    q, k, v = tokens(kv, n, 9)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out, lse, scratch = kv.new_tree_outputs(n)
    kv.tree_attend(q, k, v, i32(parents), out, lse, scratch)
    before, states = kv.export_state(), ref.state(kv)
    big = 2 ** 31 - 1
    paths = [[1, 2, -1], [0, 2, -1], [0, 1, 6], [0, 0, 1], [4, 5, -1], [-1, 0, 1], [big, -big, 0], [0, 1, 2]]
    lengths = [2, 2, 3, 2, 2, 1, 3, 4]
    retained, nret = kv.new_outputs()[1:3]
    evicted, status = i32([[[9] * 3] * 2] * 8), i32([9] * 8)
    kv.tree_commit(q, k, v, i32(parents), lse, i32(paths), i32(lengths), retained, nret, evicted, status)
    assert status.tolist() == [binding.TREEKV_EINVAL] * 8 and bool((evicted == -1).all())
    assert torch.equal(before, kv.export_state())
    assert all(retained[u // 2, u % 2].tolist() == states[u]["pos"] for u in range(16)) and bool((nret == 48).all())
    lengths = [-1, 0, big, 0, -big, 0, 1, 2]
    kv.tree_commit(q, k, v, i32(parents), lse, i32(paths), i32(lengths), retained, nret, evicted, status)
    assert status.tolist() == [-1, 0, -1, 0, -1, 0, -1, 0]
    after = ref.state(kv)
    assert [after[2 * b]["t"] - states[2 * b]["t"] for b in range(8)] == [0] * 7 + [2]
    assert evicted[7, 0].tolist()[2] == -1 and evicted[7, 0].tolist()[0] >= 0


def test_graph_replays(binding):
    """The two calls captured once and replayed as the state advances, with eager work between the replays."""
    import torch

    kv, twin = [make(binding, budget=96, batch=2, hkv=2, G=4, d=128, fed=90) for _ in range(2)]
    n, longest = 20, 4
    q, k, v = tokens(kv, n, 30)
    parents = torch.tensor([[i - 1 for i in range(n)]] * 2, dtype=torch.int32, device="cuda")
    path = torch.arange(longest, dtype=torch.int32, device="cuda").repeat(2, 1)
    lengths = torch.tensor([4, 2], dtype=torch.int32, device="cuda")
    made = []
    for c in (kv, twin):
        out, lse, scratch = c.new_tree_outputs(n)
        r, nr = c.new_outputs()[1:3]
        made.append((out, lse, scratch, r, nr, torch.empty(2, 2, longest, dtype=torch.int32, device="cuda")))

    def go(c, m):
        c.tree_attend(q, k, v, parents, *m[:3])
        c.tree_commit(q, k, v, parents, m[1], path, lengths, m[3], m[4], m[5])

    go(kv, made[0])
    go(twin, made[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(kv, made[0])
    for r in range(6):
        for x, y in zip((q, k, v), tokens(kv, n, 31 + r)):
            x.copy_(y)
        lengths.copy_(torch.tensor([r % 5, 4 - r % 5]))
        graph.replay()
        go(twin, made[1])
        torch.cuda.synchronize()
        for i in (0, 1, 3, 4, 5):
            assert torch.equal(made[0][i], made[1][i]), (r, i)
        assert torch.equal(kv.export_state(), twin.export_state())


def test_another_stream_and_shared_scratch(binding):
    """Two contexts take turns with one scratch on a stream that is not the default one."""
    import torch

    a, b = make(binding, budget=600, batch=1, fed=700), make(binding, budget=600, batch=1, fed=900, seed=2)
    n = 24
    parents = torch.tensor([[i - 1 for i in range(n)]], dtype=torch.int32, device="cuda")
    want, outs = [], []
    for kv in (a, b):
        q, k, v = tokens(kv, n, 40)
        o, lse, _ = kv.new_tree_outputs(n)
        kv.tree_attend(q, k, v, parents, o, lse)
        want.append((q, k, v, o, lse))
        outs.append(kv.new_tree_outputs(n))
    scratch = outs[0][2]
    assert scratch is not None
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            for kv, w, o in zip((a, b), want, outs):
                kv.tree_attend(*w[:3], parents, o[0], o[1], scratch)
    side.synchronize()
    for w, o in zip(want, outs):
        assert torch.equal(w[3], o[0]) and torch.equal(w[4], o[1])


def test_scratch_refused_and_outputs_bounded(binding):
    import torch

    kv = make(binding, budget=600, batch=1, fed=700)
    n, c = 10, kv.cfg
    need = kv.tree_scratch_bytes(n)
    assert need > 0 and kv.tree_scratch_bytes(0) == 0 and kv.tree_scratch_bytes(257) == 0
    q, k, v = tokens(kv, n, 41)
    parents = torch.zeros(1, n, dtype=torch.int32, device="cuda") - 1
    out, lse, scratch = kv.new_tree_outputs(n)
    with pytest.raises(binding.TreeKVError) as e:
        kv.tree_attend(q, k, v, parents, out, lse, scratch[:need - 256])
    assert e.value.status == binding.TREEKV_EINVAL
    for bad in (dict(q=q[:, :5]), dict(k=k.float()), dict(v=v.transpose(1, 2)), dict(parents=parents.long()), dict(out=out.half())):
        with pytest.raises(ValueError):
            kv.tree_attend(**{**dict(q=q, k=k, v=v, parents=parents, out=out, lse=lse), **bad})
    # what lies behind the outputs and the scratch stays as it was
    def framed(shape, dtype):
        size = torch.Size(shape).numel()
        whole = torch.full((size + 256,), 3, dtype=dtype, device="cuda")
        return whole, whole[128:128 + size].view(shape)
    frames = [framed(out.shape, out.dtype), framed(lse.shape, lse.dtype), framed((need,), torch.uint8)]
    kv.tree_attend(q, k, v, parents, *[f[1] for f in frames])
    for whole, _ in frames:
        assert bool((whole[:128] == 3).all()) and bool((whole[-128:] == 3).all())


def test_large_offsets(binding):
    """A cache whose rows pass 4 GiB: the last unit's rows are read and written where they are."""
    import torch

    kv = binding.TreeKV(70000, 1, 128, kv_heads=1, batch=260, n_sink=4, n_recent=1000, max_chunk=64)
    assert kv.workspace.numel() > 2 * (1 << 32)
    one = binding.TreeKV(70000, 1, 128, kv_heads=1, batch=1, n_sink=4, n_recent=1000, max_chunk=64)
    feed(one, 192, 3)
    kv.fork(one, [0], [259])
    n = 9
    q, k, v = tokens(one, n, 50)
    parents = [[i - 1 for i in range(n)]]
    out, retained, nret, evicted, status = run_commit(one, q, k, v, parents, [[0, 1, 2]], 3)
    big = [torch.zeros(260, *x.shape[1:], dtype=x.dtype, device="cuda") for x in (q, k, v)]
    for x, y in zip(big, (q, k, v)):
        x[259] = y[0]
    got = run_commit(kv, *big, parents * 260, [[]] * 259 + [[0, 1, 2]], 3)
    assert torch.equal(got[2][259], nret[0]) and int(got[2][259, 0]) == 195 and bool((got[2][:259] == 0).all())
    assert torch.allclose(got[0][259], out[0], rtol=0, atol=1e-5)
    K = kv.gather_kv()[0]
    assert torch.equal(K[259, 0, :195], one.gather_kv()[0][0, 0, :195]) and bool((K[259, 0, 195:] == 0).all())
