"""GPU: a sequence that is forked over another one finds nothing of it.  The one before held infinities and NaNs in all its rows;
what replaces it is shorter than the cache, and goes on bit for bit as it does in a context that never held anything else."""
import pytest

pytestmark = pytest.mark.gpu
BUDGET = 40
STREAMS = [("bf16", 64, 1, 0), ("bf16", 128, 1, 0), ("bf16", 64, 4, 0), ("bf16", 128, 2, 8), ("bf16", 64, 1, 8), ("f32", 64, 2, 0),
           ("f32", 128, 1, 0), ("f32", 64, 1, 8)]          # dtype, head_dim, query heads a KV head, flags


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def make(binding, batch, dtype, d, G, flags, **kw):
    return binding.TreeKV(BUDGET, 2 * G, d, kv_heads=2, batch=batch, dtype=dtype, flags=flags, n_sink=2, n_recent=13, max_prompt=96, **kw)


def rows(kv, n, seed):
    """q [n, H, d], k and v [n, Hkv, d], the same for every sequence, and the same whatever the batch."""
    import torch

    c, g = kv.cfg, torch.Generator().manual_seed(seed)
    return [torch.randn(n, h, c.head_dim, generator=g).to(kv.storage_dtype).cuda() for h in (c.q_heads, c.kv_heads, c.kv_heads)]


def chunk(kv, x):
    n, outs = x[0].shape[0], kv.new_outputs(x[0].shape[0])
    kv.prefill_chunk(*[y.expand(kv.cfg.batch, *y.shape).contiguous() for y in x], n, *outs)
    return outs


def step(kv, x):
    outs = kv.new_outputs()
    kv.decode_step(*[y.expand(kv.cfg.batch, *y.shape[1:]).contiguous() for y in x], *outs)
    return outs


def spoil(kv):
    """Every row of the cache, the free one too, holds values that are not finite."""
    for i, n in enumerate((BUDGET, 9, 11, 10)):
        q, k, v = rows(kv, n, i)
        k[:], v[:] = float("nan"), float("inf")
        v[::2] = float("nan")
        chunk(kv, (q, k, v))


def follow(binding, kv, fresh, seqs, kind):
    """What comes next, in both; `seqs`: the replaced sequences of `kv` and their like in `fresh`."""
    import torch

    def same(a, b, what):
        for name, x, y in zip(("out", "retained", "n_retained", "evicted"), a, b):
            for i, j in seqs:
                if name == "out":
                    assert bool(torch.isfinite(x[i]).all()), (what, name, i)
                assert torch.equal(x[i], y[j]), (what, name, i)

    for t in range(60 if kind == "steps" else 3):
        x = rows(kv, 1 if kind == "steps" else (5, 40, 33)[t], 700 + t)
        call = step if kind == "steps" else chunk
        same(call(kv, x), call(fresh, x), (kind, t))
    a, b = kv.gather_kv(), fresh.gather_kv()
    for i, j in seqs:
        assert torch.equal(kv.scores()[i], fresh.scores()[j]) and torch.equal(a[0][i], b[0][j]) and torch.equal(a[1][i], b[1][j])


@pytest.mark.parametrize("kind", ["steps", "chunks"])
@pytest.mark.parametrize("fed", [1, 17, 39])
@pytest.mark.parametrize("stream", STREAMS, ids=str)
def test_fork(binding, stream, fed, kind):
    import torch

    kv, source, empty = [make(binding, b, *stream, kv_splits=1) for b in (4, 1, 1)]
    spoil(kv)
    chunk(source, rows(source, fed, 2))
    kv.fork(source, [0, -1], [2, 1])
    assert not torch.isfinite(kv.gather_kv()[1][0].float()).any()
    follow(binding, kv, source, [(2, 0)], kind)
    # (the emptied one has followed too)
    for t in range(60 if kind == "steps" else 3):
        x = rows(empty, 1 if kind == "steps" else (5, 40, 33)[t], 700 + t)
        (step if kind == "steps" else chunk)(empty, x)
    a, b = kv.gather_kv(), empty.gather_kv()
    assert torch.equal(kv.scores()[1], empty.scores()[0]) and torch.equal(a[0][1], b[0][0]) and torch.equal(a[1][1], b[1][0])


@pytest.mark.parametrize("kind", ["steps", "chunks"])
@pytest.mark.parametrize("stream", STREAMS, ids=str)
def test_emptied(binding, stream, kind):
    kv, fresh = make(binding, 3, *stream, kv_splits=1), make(binding, 1, *stream, kv_splits=1)
    spoil(kv)
    kv.fork(kv, [-1, -1], [2, 0])
    follow(binding, kv, fresh, [(2, 0), (0, 0)], kind)
