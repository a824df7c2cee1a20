"""GPU: drafted trees over caches of every layout (no sinks, no recent window, a tree region of one slot, a budget of one), rounds of
attention and commit against the plain 64-bit forms, and the largest number of units."""
import random

import pytest

from tests import speculate_reference as ref
from tests.test_gpu_tree import binding, check_attend, run_commit, tokens  # noqa: F401 (binding: the fixture)

pytestmark = pytest.mark.gpu
RERANK = 8

LAYOUTS = [
    # budget, sinks, recent
    (1, 0, 0), (2, 1, 0), (3, 1, 1), (9, 0, 0), (9, 0, 8), (9, 8, 0), (33, 0, 12), (33, 5, 0), (64, 31, 32), (40, 3, 11),
]


@pytest.mark.parametrize("dtype,d,G,flags", [("bf16", 64, 1, 0), ("bf16", 128, 8, 0), ("f32", 64, 2, 0), ("bf16", 128, 1, RERANK),
                                             ("bf16", 64, 8, RERANK), ("f32", 128, 4, RERANK), ("f32", 128, 8, 4), ("bf16", 64, 2, 1)])
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda x: "-".join(map(str, x)))
def test_rounds(binding, layout, dtype, d, G, flags):  # noqa: F811
    import torch

    budget, sinks, recent = layout
    kv = binding.TreeKV(budget, 2 * G, d, kv_heads=2, batch=2, dtype=dtype, flags=flags, n_sink=sinks, n_recent=recent, max_chunk=50)
    rng = random.Random(budget * 100 + sinks)
    for rnd in range(4):
        n = rng.choice([1, 3, 17, 50])
        longest = rng.randint(1, min(n, 20))
        parents, paths = [], []
        for b in range(2):
            nodes = sorted(rng.sample(range(n), rng.randint(0, longest)))
            p = [rng.randint(-1, i - 1) if i else -1 for i in range(n)]
            for x, node in enumerate(nodes):
                p[node] = nodes[x - 1] if x else -1
            parents.append(p), paths.append(nodes)
        q, k, v = tokens(kv, n, 900 + rnd)
        before = ref.state(kv)
        out, lse, scratch = kv.new_tree_outputs(n)
        kv.tree_attend(q, k, v, torch.tensor(parents, dtype=torch.int32, device="cuda"), out, lse, scratch)
        check_attend(kv, q, k, v, parents, out, lse)
        _, retained, nret, evicted, status = run_commit(kv, q, k, v, parents, paths, longest)
        assert status.tolist() == [0, 0]
        after = ref.state(kv)
        qd, kd, vd = [x.double().cpu() for x in (q, k, v)]
        for b in range(2):
            for h in range(2):
                u = b * 2 + h
                args = (qd[b, :, h * G:(h + 1) * G], kd[b, :, h], vd[b, :, h], parents[b])
                want, gone, margin = ref.commit_unit(kv, before[u], *args, paths[b])
                got = after[u]
                if margin > 1e-5:                          # (fp32 scores are off by some 1e-6: nearer pairs may go either way)
                    assert evicted[b, h].tolist() == gone + [-1] * (longest - len(gone)), (rnd, b, h)
                    assert (got["n"], got["t"], got["idx"], got["pos"]) == (want["n"], want["t"], want["idx"], want["pos"]), (rnd, b, h)
                    assert torch.equal(got["K"], want["K"]) and torch.equal(got["V"], want["V"])
                    bound = float(ref.attend_unit(kv, before[u], *args)[3].max()) if paths[b] else 0.0
                    room = (bound + (len(paths[b]) * G + 4) * 2.0 ** -24) * want["S"] + 2.0 ** -120
                    assert bool(((got["S"] - want["S"]).abs() <= room).all()), (rnd, b, h)
                assert retained[b, h].tolist() == got["pos"] + [-1] * (budget - got["n"]) and int(nret[b, h]) == got["n"]
                assert got["n"] == min(budget, before[u]["n"] + len(paths[b])) and got["t"] == before[u]["t"] + len(paths[b])


@pytest.mark.parametrize("flags", [0, RERANK])
def test_the_largest_number_of_units(binding, flags):  # noqa: F811
    """65535 units: the last one's results are those of a context of its own."""
    import torch

    U, n, path = 65535, 5, [0, 1, 3]
    parents = [-1, 0, 1, 1, 2]
    kw = dict(kv_heads=1, n_sink=1, n_recent=4, max_chunk=16, flags=flags, kv_splits=1)
    kv, one = binding.TreeKV(16, 1, 64, batch=U, **kw), binding.TreeKV(16, 1, 64, batch=1, **kw)
    for rnd in range(6):
        q, k, v = tokens(one, n, 60 + rnd)
        got = run_commit(one, q, k, v, [parents], [path], 3)
        big = [x.expand(U, -1, -1, -1).contiguous() for x in (q, k, v)]
        many = run_commit(kv, *big, [parents] * U, [path] * U, 3)
        for x, y in zip(many[1:4], got[1:4]):
            assert torch.equal(x[-1], y[0]) and torch.equal(x[0], y[0]) and torch.equal(x[U // 2], y[0])
        assert bool((many[4] == 0).all()) and bool((many[0] == many[0][:1]).all())
        assert torch.allclose(many[0][-1], got[0][0], rtol=0, atol=1e-5)       # (another number of slices)
    kv.fork(one, [-1] * 3 + [0], [0, 1, U // 2, U - 1])
    assert torch.equal(kv.gather_kv()[0][-1], one.gather_kv()[0][0]) and torch.equal(kv.scores()[-1], one.scores()[0])
    state = kv.export_state()
    twin = binding.TreeKV(16, 1, 64, batch=U, **kw)
    twin.import_state(state)
    assert torch.equal(twin.export_state(), state)
