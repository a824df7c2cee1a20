"""GPU: treekv_qkv_prepare against its formula in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def reference(x, w, eps, positions, freq, rot, halves, to_planes):
    """-> (value, size): what comes out, and the size of the terms each value is made of."""
    import torch

    y = x.double()
    if w is not None:
        y = y / (y.square().mean(dim=-1, keepdim=True) + eps).sqrt() * w.double()
    out, size, h = y.clone(), y.abs(), rot // 2
    if rot:
        first = torch.arange(h) if halves else 2 * torch.arange(h)
        second = first + h if halves else first + 1
        angle = positions.double()[:, None, None] * freq if positions is not None else torch.zeros(1, 1, h, dtype=torch.float64)
        a, b = y[..., first], y[..., second]
        where = (2 * torch.arange(h), 2 * torch.arange(h) + 1) if to_planes else (first, second)
        out[..., where[0]], out[..., where[1]] = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
        size[..., where[0]] = size[..., where[1]] = a.abs() + b.abs()
    return out, size


def check(got, want, size, dtype, d):
    import torch

    # One rounding to the storage type: half a step, eps / 2 of the value.  Before it, in fp32: the sum of squares (d / lanes
    # products and the tree over the lanes, 20 roundings at most), the root, the two products, the sine and cosine (two steps
    # each and 3 for their angle) and the turn: 40 roundings of 2^-24 of the terms' size at most.
    half = torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0
    room = half * want.abs() + (1 + half) * 40 * 2.0 ** -24 * size + 1e-37
    off = (got.double().cpu() - want).abs()
    assert bool((off <= room).all()), float((off / room).max())


CASES = [(t, d, hq, hkv, dt) for t, hq, hkv in ((1, 32, 8), (3, 1, 1), (67, 5, 3)) for d in (64, 128) for dt in ("bfloat16", "float32")]


@pytest.mark.parametrize("rot", [0, 16, 48, 64, "all"])
@pytest.mark.parametrize("mode", ["pairs", "halves", "planes"])
@pytest.mark.parametrize("tokens,d,hq,hkv,dt", CASES)
def test_packed_rows(binding, tokens, d, hq, hkv, dt, mode, rot):
    import torch

    dtype, rot = getattr(torch, dt), d if rot == "all" else rot
    halves, planes = mode != "pairs", mode == "planes"
    g = torch.Generator().manual_seed(tokens * d + hq)
    qkv = (torch.randn(tokens, (hq + 2 * hkv) * d, generator=g) * 3).to(dtype)
    qw, kw = [(1 + 0.3 * torch.randn(d, generator=g)).to(dtype) for _ in range(2)]
    positions = torch.randint(-5, 1 << 20, (tokens,), generator=g).int() if rot else None
    freq = binding.rope_frequencies(rot, 500000.0, device="cpu") if rot else None
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    packed = qkv.cuda()
    q, k, v = [x.unflatten(1, (-1, d)) for x in packed.split([hq * d, hkv * d, hkv * d], dim=1)]
    for weights in ((qw, kw), (None, kw), (None, None)):
        got = binding.qkv_prepare(q, k, v, q_weight=dev(weights[0]), k_weight=dev(weights[1]), eps=1e-5, positions=dev(positions),
                                  inv_freq=dev(freq), halves=halves, to_planes=planes)
        r = rot if rot or not planes else d              # without positions the planes of the whole head are written in order
        for x, y, w in ((q, got[0], weights[0]), (k, got[1], weights[1])):
            want, size = reference(x.cpu(), w, 1e-5, positions, freq, r, halves, planes)
            assert y.is_contiguous() and y.shape == x.shape
            check(y, want, size, dtype, d)
        assert torch.equal(got[2], v)
    assert torch.equal(packed.cpu(), qkv)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("mode", ["pairs", "halves", "planes"])
def test_in_place_and_parts(binding, dt, mode):
    import torch

    dtype = getattr(torch, dt)
    q = torch.randn(300, 9, 128, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    w = torch.ones(128, dtype=dtype, device="cuda")
    kw = dict(q_weight=w, positions=torch.arange(300, device="cuda").int(), inv_freq=binding.rope_frequencies(128),
              halves=mode != "pairs", to_planes=mode == "planes")
    want = binding.qkv_prepare(q, **kw)[0]
    both = binding.qkv_prepare(q, q[:, :2], None, k_weight=w, **kw)
    assert torch.equal(both[0], want) and torch.equal(both[1], want[:, :2]) and both[2] is None
    only = binding.qkv_prepare(None, None, q)
    assert torch.equal(only[2], q)
    y = q.clone()
    assert binding.qkv_prepare(y, out=(y, None, None), **kw)[0] is y and torch.equal(y, want)


def test_values_at_the_edges(binding):
    """Zeros, the smallest and the largest values; a NaN stays in its head; negative zero and NaN bits of v are copied."""
    import torch

    x = torch.randn(8, 4, 64, generator=torch.Generator().manual_seed(2)).bfloat16()
    x[0] = 0.0
    x[1] = 1e-30
    x[2, 1, 5] = float("nan")
    x[3] *= 1e15
    x[4, 0, 0] = float("inf")
    w = torch.ones(64, dtype=torch.bfloat16)
    q, _, v = binding.qkv_prepare(x.cuda(), x.cuda(), x.cuda(), q_weight=w.cuda(), eps=1e-6)
    q = q.cpu()
    assert bool((q[0] == 0).all()) and bool(torch.isnan(q[2, 1]).all()) and bool(torch.isfinite(q[2, [0, 2, 3]]).all())
    assert torch.equal(v.cpu().view(torch.int16), x.view(torch.int16))
    for i in (1, 3, 5):
        want, size = reference(x[i:i + 1], w, 1e-6, None, None, 0, False, False)
        check(q[i:i + 1], want, size, torch.bfloat16, 64)


def test_many_tokens(binding):
    """More rows than 32 bits of elements hold: the last token's are where they should be."""
    import torch

    tokens, h = 1 << 19, 33
    q = torch.empty(tokens, h, 128, dtype=torch.bfloat16, device="cuda")
    assert q.numel() > 1 << 31
    q.fill_(0.5)
    q[-1] = torch.arange(128, device="cuda").to(torch.bfloat16)
    out = binding.qkv_prepare(q, q_weight=torch.ones(128, dtype=torch.bfloat16, device="cuda"), eps=0.0)[0]
    assert bool((out[:-1:1001] == 1.0).all()) and bool((out[-2] == 1.0).all())
    want, size = reference(q[-1:].cpu(), torch.ones(128), 0.0, None, None, 0, False, False)
    check(out[-1:], want, size, torch.bfloat16, 128)


def test_stream_and_graph(binding):
    import torch

    q = torch.randn(40, 6, 128, device="cuda").bfloat16()
    pos = torch.arange(40, device="cuda").int()
    kw = dict(inv_freq=binding.rope_frequencies(128), positions=pos)
    out = (torch.empty_like(q), None, None)
    want = binding.qkv_prepare(q, **kw)[0]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.qkv_prepare(q, out=out, **kw)
    for r in range(4):
        pos += 1
        q.mul_(0.5)
        want = binding.qkv_prepare(q, **kw)[0]
        graph.replay()
        assert torch.equal(out[0], want), r
        out[0].zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = binding.qkv_prepare(q, **kw)[0]
    side.synchronize()
    assert torch.equal(got, want)


def test_into_a_cache_with_reassigned_positions(binding):
    """A model that pairs halves: its turned operands in a plain context attend as its permuted ones do in a context that turns
    them itself, while nothing has been evicted."""
    import torch

    hq, hkv, d, n = 4, 2, 64, 40
    plain = binding.TreeKV(64, hq, d, kv_heads=hkv, dtype="f32", n_sink=2, n_recent=20)
    turned = binding.TreeKV(64, hq, d, kv_heads=hkv, dtype="f32", n_sink=2, n_recent=20, flags=binding.TREEKV_POSITION_RERANK)
    rows = torch.randn(n, (hq + 2 * hkv) * d, generator=torch.Generator().manual_seed(1)).cuda()
    q, k, v = [x.unflatten(1, (-1, d)) for x in rows.split([hq * d, hkv * d, hkv * d], dim=1)]
    a = binding.qkv_prepare(q, k, v, positions=torch.arange(n, device="cuda").int(), inv_freq=binding.rope_frequencies(d), halves=True)
    b = binding.qkv_prepare(q, k, v, halves=True, to_planes=True)
    outs = []
    for kv, x in ((plain, a), (turned, b)):
        o, r, nr, ev = kv.new_outputs(n)
        kv.prefill_chunk(*[y[None] for y in x], n, o, r, nr, ev)
        outs.append(o)
    # logits of size 8 at most, d + 20 roundings each, in either context
    assert torch.allclose(outs[0], outs[1], rtol=0, atol=2 * 2 * 84 * 2.0 ** -24 * 64)


@pytest.mark.parametrize("dt", ["bfloat16", "float32"])
@pytest.mark.parametrize("d", [64, 128])
def test_order_of_planes_alone(binding, dt, d):
    """Neither normalised nor turned: the halves' pairs side by side, every value as it was, infinities and the largest too."""
    import torch

    dtype = getattr(torch, dt)
    x = torch.randn(5, 3, d, generator=torch.Generator().manual_seed(d)).to(dtype)
    x[0, 0, 3], x[1, 1, d // 2 + 3], x[2, 2, 7], x[3, 0, d - 1] = float("inf"), -float("inf"), torch.finfo(dtype).max, -0.0
    got = binding.qkv_prepare(x.cuda(), x.cuda(), x.cuda(), halves=True, to_planes=True)
    want = torch.stack([x[..., :d // 2], x[..., d // 2:]], dim=-1).flatten(-2)
    for y in got[:2]:
        assert torch.equal(y.cpu().view(torch.uint8), want.contiguous().view(torch.uint8))
    assert torch.equal(got[2].cpu(), x)
