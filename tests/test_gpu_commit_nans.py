"""GPU: NaNs among the operands of treekv_tree_commit."""
import random

import pytest

from tests import speculate_reference as ref
from tests.test_gpu_tree import binding, make, tokens  # noqa: F401 (binding: the fixture)

pytestmark = pytest.mark.gpu
RERANK = 8


@pytest.mark.parametrize("where", ["key", "query", "lse"])
@pytest.mark.parametrize("fed", [30, 133])
@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("f32", 0), ("bf16", RERANK), ("f32", RERANK)])
def test_a_nan_adds_nothing(binding, dtype, flags, fed, where):  # noqa: F811
    """A NaN among a path's operands makes NaNs of probabilities; they add nothing, and all others add what they are."""
    import torch

    G, n, bad = 2, 9, 3
    kv = make(binding, budget=48, batch=2, hkv=2, G=G, d=64, dtype=dtype, flags=flags, fed=fed)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rng = random.Random(4)
    parents = [[i - 1 for i in range(6)] + [rng.randint(-1, 5) for _ in range(n - 6)] for _ in range(2)]
    paths = [list(range(6))] * 2
    q, k, v = tokens(kv, n, 85)
    out, lse, scratch = kv.new_tree_outputs(n)
    kv.tree_attend(q, k, v, i32(parents), out, lse, scratch)
    before = ref.state(kv)
    qd, kd, vd = [x.double().cpu() for x in (q, k, v)]
    # of sequence 0, KV head 1: the rows (node, head of the group) whose probabilities are NaNs
    if where == "key":                                     # the node's descendants and itself attend it
        k[0, bad, 1, 5] = float("nan")
        lost = {(i, g) for i in range(bad, 6) for g in range(G)}
    elif where == "query":
        q[0, bad, 3, 7] = float("nan")
        lost = {(bad, 1)}
    else:
        lost = {(bad, 0), (bad, 1)}
    kv.tree_attend(q, k, v, i32(parents), out, lse, scratch)
    if where == "lse":
        lse[0, bad, 2:] = float("nan")
    retained, nret = kv.new_outputs()[1:3]
    status, evicted = i32([9, 9]), i32([[[9] * 6] * 2] * 2)
    kv.tree_commit(q, k, v, i32(parents), lse, i32(paths), i32([6, 6]), retained, nret, evicted, status)
    assert status.tolist() == [0, 0]
    for u, (old, new) in enumerate(zip(before, ref.state(kv))):
        b, h = divmod(u, 2)
        args = (qd[b, :, h * G:(h + 1) * G], kd[b, :, h], vd[b, :, h], parents[b])
        probs, bound = [ref.attend_unit(kv, old, *args)[i] for i in (4, 3)]
        score = old["S"].tolist() + [0.0] * 6
        for x, node in enumerate(paths[b]):
            for g in range(G):
                if (b, h) == (0, 1) and (x, g) in lost:
                    continue
                for j, p in enumerate(probs[node][g].tolist()):
                    score[j] += p
        where_at = old["pos"] + [old["t"] + i for i in range(6)]
        want = torch.tensor([score[where_at.index(x)] for x in new["pos"]], dtype=torch.float64)
        room = (float(bound.max()) + (6 * G + 4) * 2.0 ** -24) * want
        assert bool(((new["S"] - want).abs() <= room).all()), (u, float((new["S"] - want).abs().max()))
        assert int(nret[b, h]) == new["n"] == min(48, old["n"] + 6)
