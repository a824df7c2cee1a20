"""GPU: treekv_tree_attend over caches that hold far fewer tokens than they have room for.  Slices are counted by the room, so
that some of them have no column at all; what they leave to the merge is nothing."""
import random

import pytest

from tests.test_gpu_tree import binding, check_attend, make, tokens, tree  # noqa: F401 (binding: the fixture)

pytestmark = pytest.mark.gpu
RERANK = 8


# (tokens cached, of 2048): none, one, one tile of 64 columns, a little more
@pytest.mark.parametrize("fed", [0, 1, 64, 70])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,hkv,G,nodes,dtype,flags", [
    (16, 4, 4, 13, "bf16", RERANK),                        # 64 units x 52 rows: keys turned for 64 rows, eight slices
    (2, 2, 2, 9, "bf16", RERANK),
    (8, 8, 4, 40, "bf16", 0),                              # 160 rows a unit, tiles shared by 128
    (1, 2, 4, 7, "bf16", 0),
    (1, 2, 2, 9, "f32", RERANK),
])
def test_slices_without_columns(binding, batch, hkv, G, nodes, dtype, flags, d, fed):  # noqa: F811
    import torch

    kv = make(binding, budget=2048, batch=batch, hkv=hkv, G=G, d=d, dtype=dtype, flags=flags, fed=fed, seed=fed + 3)
    rng = random.Random(nodes)
    parents = [tree("drafted", nodes, rng) for _ in range(batch)]
    q, k, v = tokens(kv, nodes, 91)
    out, lse, scratch = kv.new_tree_outputs(nodes)
    assert scratch is not None                             # several slices
    scratch.fill_(255)                                     # (NaNs)
    par = torch.tensor(parents, dtype=torch.int32, device="cuda")
    kv.tree_attend(q, k, v, par, out, lse, scratch)
    check_attend(kv, q, k, v, parents, out, lse, every=1 if batch * hkv < 20 else 13)
    again = torch.empty_like(out)
    kv.tree_attend(q, k, v, par, again)
    assert torch.equal(out, again)
