"""GPU: what treekv_tree_commit adds to the scores where the sums are tiny."""
import pytest

from tests import speculate_reference as ref
from tests.test_gpu_tree import binding, make, run_commit, tokens  # noqa: F401 (binding: the fixture)

pytestmark = pytest.mark.gpu
RERANK = 8


def without_scores(kv):
    """The context's scores set to 0, so that a commit's own sums are what comes out."""
    import torch

    buf, lay, c = kv.export_state(), kv.state_layout(), kv.cfg
    ref.part(buf, lay.S, torch.float32, c.batch * c.kv_heads, c.budget).zero_()
    kv.import_state(buf)


@pytest.mark.parametrize("path", [1, 2, 40])
@pytest.mark.parametrize("dtype,d,G,flags", [("bf16", 64, 1, 0), ("bf16", 128, 4, 0), ("f32", 64, 2, 0), ("f32", 128, 1, 0),
                                             ("bf16", 128, 2, RERANK), ("f32", 64, 8, RERANK)])
def test_tiny_sums(binding, dtype, d, G, flags, path):  # noqa: F811
    """Probabilities between 1 and 2^-100: each column's sum is as exact as its probabilities are."""
    import torch

    kv = make(binding, budget=200, batch=1, hkv=2, G=G, d=d, dtype=dtype, flags=flags, fed=150, seed=path)
    without_scores(kv)
    q, k, v = tokens(kv, path, 83, scale=6.0)
    before = ref.state(kv)
    parents = [i - 1 for i in range(path)]
    assert run_commit(kv, q, k, v, [parents], [list(range(path))], path)[4].tolist() == [0]
    qd, kd, vd = [x.double().cpu() for x in (q, k, v)]
    tiny = 0
    for h, (old, new) in enumerate(zip(before, ref.state(kv))):
        args = (qd[0, :, h * G:(h + 1) * G], kd[0, :, h], vd[0, :, h], parents)
        want = ref.commit_unit(kv, old, *args, list(range(path)))[0]["S"]
        # a probability is off by what its logits are (see attend_unit), the sum by a rounding of 2^-24 each; below 2^-126 an
        # exponential is 0
        bound = float(ref.attend_unit(kv, old, *args)[3].max())
        room = (bound + (path * G + 4) * 2.0 ** -24) * want + path * G * 2.0 ** -126
        off = (new["S"] - want).abs()
        assert bool((off <= room).all()), (h, float((off / room).max()))
        tiny += int((want < 2.0 ** -24).sum())
    assert path * G > 8 or tiny > 10                       # (some are)


@pytest.mark.parametrize("flags", [0, RERANK])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_as_a_step(binding, dtype, flags):  # noqa: F811
    """A path of one token adds what a decode step adds, in the tail too."""
    import torch

    kw = dict(budget=200, batch=1, hkv=2, G=2, d=64, dtype=dtype, flags=flags, fed=150)
    kv, twin = make(binding, **kw), make(binding, **kw)
    without_scores(kv), without_scores(twin)
    q, k, v = tokens(kv, 1, 84, scale=6.0)
    run_commit(kv, q, k, v, [[-1]], [[0]], 1)
    twin.decode_step(*[x[:, 0].contiguous() for x in (q, k, v)], *twin.new_outputs())
    a, b = kv.scores().double()[:, :, :151], twin.scores().double()[:, :, :151]
    assert float(b.min()) < 2.0 ** -30
    # logits below 2^7 in units of log2: 64 products, the scale and (re-assigned) the turning of both sides are some 80 roundings
    # of 2^-24 of the products' sizes (below 2^8) on either side, the lse two more: 2 * 82 * 2^-16 * ln 2 of the probability
    assert bool(((a - b).abs() <= 2 * 82 * 2.0 ** -16 * 0.7 * b + 2.0 ** -125).all()), float(((a - b).abs() / b).max())
