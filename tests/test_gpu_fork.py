"""GPU: treekv_fork.  A copy's whole state is its source's, it goes on bit for bit as its source does, and nothing else moves."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def make(binding, batch, *, budget=40, hkv=2, G=2, d=64, dtype="bf16", flags=0, **kw):
    return binding.TreeKV(budget, hkv * G, d, kv_heads=hkv, batch=batch, dtype=dtype, flags=flags, n_sink=2, n_recent=budget // 3, **kw)


def step(kv, seed, same=False):
    """A decode step on random tokens (the same ones for every sequence)."""
    import torch

    c, g = kv.cfg, torch.Generator().manual_seed(seed)
    x = [torch.randn(1 if same else c.batch, h, c.head_dim, generator=g).expand(c.batch, -1, -1).contiguous().to(kv.storage_dtype).cuda()
         for h in (c.q_heads, c.kv_heads, c.kv_heads)]
    outs = kv.new_outputs()
    kv.decode_step(*x, *outs)
    return outs


def parts(kv):
    """{name: [B, Hkv, ..]} of the state, on the host."""
    import torch

    from tests import speculate_reference as ref

    c, lay, buf = kv.cfg, kv.state_layout(), kv.export_state().cpu()
    dt, shape = kv.storage_dtype, (c.batch, c.kv_heads, c.budget)
    return dict(header=ref.part(buf, lay.header, torch.int32, *shape[:2], 4), pos=ref.part(buf, lay.positions, torch.int32, *shape),
                slots=ref.part(buf, lay.slots, torch.int32, *shape), S=ref.part(buf, lay.S, torch.float32, *shape),
                K=ref.part(buf, lay.K, dt, *shape, c.head_dim), V=ref.part(buf, lay.V, dt, *shape, c.head_dim))


@pytest.mark.parametrize("fed", [0, 1, 25, 40, 170])
@pytest.mark.parametrize("dtype,d,flags,kw", [("bf16", 64, 0, {}), ("f32", 128, 0, dict(budget=33)), ("bf16", 128, 8, dict(kv_splits=3))])
def test_between_contexts(binding, fed, dtype, d, flags, kw):
    import torch

    source, to = make(binding, 3, d=d, dtype=dtype, flags=flags, **kw), make(binding, 5, d=d, dtype=dtype, flags=flags, **{**kw, "kv_splits": 1})
    for t in range(fed):
        step(source, t)
    for t in range(60):
        step(to, 1000 + t)
    was, src = parts(to), parts(source)
    to.fork(source, [2, 0, -1, 2], [4, 1, 0, 2])
    now = parts(to)
    empty = dict(header=torch.tensor([0, 0, 1, 0], dtype=torch.int32), pos=-1, slots=-1, S=0, K=0, V=0)
    for name in now:
        for dst, s in ((4, 2), (1, 0), (2, 2)):
            assert torch.equal(now[name][dst], src[name][s]), (name, dst)
        assert bool((now[name][0] == empty[name]).all()), name
        assert torch.equal(now[name][3], was[name][3]), name
    # what follows: the copies of a sequence evict and score as their source, which keeps its own state
    for t in range(70):
        a, b = step(source, 5000 + t, same=True), step(to, 5000 + t, same=True)
        for x, y in zip(a[1:], b[1:]):
            assert torch.equal(y[4], x[2]) and torch.equal(y[2], x[2]) and torch.equal(y[1], x[0])
        if "kv_splits" not in kw:
            assert torch.equal(a[0][2], b[0][4])
    assert torch.equal(parts(source)["pos"][0], parts(to)["pos"][1])


def test_inside_a_context(binding):
    import torch

    kv = make(binding, 70, hkv=1, G=1)
    for t in range(55):
        step(kv, t)
    was = parts(kv)
    src, dst = [3] * 60 + [1, 2, -1], list(range(10, 70)) + [1, 4, 0]          # one stays itself; more pairs than a launch holds
    kv.fork(kv, src, dst)
    now = parts(kv)
    for name in now:
        for s, x in zip(src, dst):
            if s >= 0:
                assert torch.equal(now[name][x], was[name][s])
        for x in (2, 3, 5, 6, 7, 8, 9):
            assert torch.equal(now[name][x], was[name][x])
    assert now["header"][0, 0].tolist() == [0, 0, 1, 0]
    before = kv.export_state()
    for bad in (([3], [70]), ([70], [3]), ([-2], [3]), ([3], [-1]), ([1, 2], [5, 5]), ([1, 5], [5, 6]), ([], []), ([1] * 71, list(range(70)) + [0])):
        with pytest.raises(binding.TreeKVError) as e:
            kv.fork(kv, *bad)
        assert e.value.status == binding.TREEKV_EINVAL
    with pytest.raises(ValueError):
        kv.fork(kv, [1], [2, 3])
    for other in (dict(budget=41), dict(hkv=2, G=1), dict(hkv=1, G=2), dict(d=128), dict(dtype="f32"), dict(flags=1), dict(softmax_scale=0.5)):
        with pytest.raises(binding.TreeKVError) as e:
            kv.fork(make(binding, 2, **{**dict(hkv=1, G=1), **other}), [0], [1])
        assert e.value.status == binding.TREEKV_EINVAL
    assert torch.equal(before, kv.export_state())
    # a second handle on the same workspace is the same context
    twin = make(binding, 70, hkv=1, G=1)
    twin._lib.treekv_bind_workspace(twin._h, kv.workspace.data_ptr(), kv.workspace.numel())
    with pytest.raises(binding.TreeKVError):
        kv.fork(twin, [1, 5], [5, 6])


def test_prompt_into_a_batch(binding):
    """A prompt compressed in a context of its own becomes the start of four samples, which then differ."""
    import torch

    one = make(binding, 1, budget=64, max_prompt=256)
    many = make(binding, 4, budget=64)
    g = torch.Generator().manual_seed(9)
    qw, k, v = [torch.randn(1, n, h, 64, generator=g).bfloat16().cuda() for n, h in ((16, 4), (256, 2), (256, 2))]
    ret = torch.empty(1, 2, 64, dtype=torch.int32, device="cuda")
    one.prefill_prompt(qw, k, v, 256, 16, ret)
    many.fork(one, [0] * 4, [0, 1, 2, 3])
    p = parts(many)
    assert all(torch.equal(p["pos"][b], ret[0].cpu()) for b in range(4))
    outs = step(many, 3)
    assert not torch.equal(outs[0][0], outs[0][1])
    assert bool((outs[2] == 64).all()) and bool((outs[3] >= 0).all())


def test_captured(binding):
    import torch

    a, b = make(binding, 2), make(binding, 3)
    for t in range(50):
        step(a, t)
    b.fork(a, [0], [0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.fork(a, [1, 0, -1], [0, 2, 1])
    for r in range(4):
        step(a, 100 + r)
        step(b, 200 + r)
        graph.replay()
        x, y = parts(a), parts(b)
        for name in x:
            assert torch.equal(x[name][1], y[name][0]) and torch.equal(x[name][0], y[name][2])
        assert int(y["header"][1, :, 0].max()) == 0
