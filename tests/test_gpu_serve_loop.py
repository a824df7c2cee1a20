"""GPU: the paged cache and the verification of drafts as a serving loop uses them, eager and captured."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def held(got, want, room):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= room).all()), float((off / room.clamp(min=1e-300)).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_chunks_appended_attended_and_evicted(binding, dtype):
    """Chunks of unequal sequences, then single tokens, each step appended, attended with its weights, and cut to the budget."""
    import torch

    from tests.serve_reference import Paged

    budget, sink, recent = 48, 4, 16
    ref = Paged(lens=[0, 0, 0], news=[0, 0, 0], page_size=16, kv_heads=2, group=3, d=64, dtype=dtype, width=8, spare=24, seed=1)
    for b in range(3):
        ref.table[b] = torch.arange(8 * b, 8 * b + 8)
    ref.weights.fill_(0.5)                                     # what a slot held before is no part of its next token's weight
    kv, seen = ref.on_gpu(binding), [0, 0, 0]
    for news in ([70, 33, 1], [9, 40, 0], [1, 1, 1], [80, 80, 80], [1, 0, 1], [1, 1, 1], [3, 64, 2]):
        starts = [0]
        for n in news:
            starts.append(starts[-1] + n)
        ref.news, ref.starts, ref.total = news, torch.tensor(starts, dtype=torch.int32), starts[-1]
        ref.lens += torch.tensor(news, dtype=torch.int32)
        kv.lens.add_(torch.tensor(news, dtype=torch.int32, device="cuda"))
        k, v = [torch.randn(ref.total, 2, 64, generator=ref.g).to(ref.t) for _ in "kv"]
        ref.q = torch.randn(ref.total, 6, 64, generator=ref.g).to(ref.t)
        positions = torch.cat([torch.arange(s, s + n) for s, n in zip(seen, news)]).int()
        kv.append(k.cuda(), v.cuda(), ref.starts.cuda(), positions.cuda())
        ref.append(k, v, positions)
        lse = torch.empty(ref.total, 6, device="cuda")
        out = kv.attend(ref.q.cuda(), ref.starts.cuda(), max(news), None, lse, weigh=True)
        want = ref.attend()
        held(out, want["out"], want["room"])
        held(lse, want["lse"], want["lse_room"])
        total = ref.weights.double() + want["gain"]
        held(kv.weights, total, want["gain_room"] + 2.0 ** -23 * total.abs())
        ref.weights.copy_(kv.weights)                          # the order of what is kept is that of these weights
        kv.evict(budget, sink, recent)
        ref.evict(budget, sink, recent)
        for name in ("k", "v", "weights", "positions", "lens"):
            assert torch.equal(getattr(kv, name).cpu(), getattr(ref, name)), name
        seen = [s + n for s, n in zip(seen, news)]
        for b in range(3):
            kept = kv.positions[b, :, :min(seen[b], budget)].cpu()
            for h in range(2):
                got = set(kept[h].tolist())
                assert set(range(min(sink, seen[b]))) <= got and set(range(max(0, seen[b] - recent), seen[b])) <= got
                assert len(got) == min(seen[b], budget)


def test_a_captured_step_replayed(binding):
    """A decode step and its eviction as a graph, beside the same steps eager; two graphs share the scratch."""
    import torch

    from tests.serve_reference import Paged

    def start():
        ref = Paged(lens=[60, 64, 20], news=[1, 1, 1], page_size=16, kv_heads=2, group=4, d=128, width=6, spare=18, seed=4)
        for b in range(3):
            ref.table[b] = torch.arange(6 * b, 6 * b + 6)
        return ref, ref.on_gpu(binding)

    ref, a = start()
    _, b = start()
    g = torch.Generator(device="cuda").manual_seed(5)
    starts = ref.starts.cuda()
    k, v = [torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    q, at = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    outs = [torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda") for _ in "ab"]
    scratch, cut = a.new_attend_scratch(3, 1, weigh=True), a.new_evict_scratch()

    def step(kv, out):
        kv.lens.add_(1)
        kv.append(k, v, starts, at)
        kv.attend(q, starts, 1, out, weigh=True, scratch=scratch)
        kv.evict(62, 2, 20, scratch=cut)

    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for kv, out in ((a, outs[0]), (b, outs[0])):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step(kv, out)
            graphs.append(graph)
    torch.cuda.synchronize()
    _, c = start()
    _, a2 = start()
    for name in ("k", "v", "weights", "positions", "lens"):
        assert torch.equal(getattr(a, name), getattr(c, name)), name                    # capturing has run nothing
    for i in range(12):
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        at.fill_(100 + i)
        graphs[i % 2].replay()
        twin = (c, a2)[i % 2]
        step(twin, outs[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]), i
        for name in ("k", "v", "weights", "positions", "lens"):
            assert torch.equal(getattr((a, b)[i % 2], name), getattr(twin, name)), (i, name)


@pytest.mark.parametrize("weigh", [False, True])
def test_captured_chunks_and_long_vocabularies(binding, weigh):
    """The kernels of many rows and the passes by several workgroups, captured and replayed beside eager calls."""
    import torch

    from tests.serve_reference import Paged

    ref = Paged(lens=[150, 260], news=[150, 90], page_size=16, kv_heads=2, group=2, d=128, seed=14)
    a, b = ref.on_gpu(binding), ref.on_gpu(binding)
    starts, q = ref.starts.cuda(), torch.zeros_like(ref.q, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(15)
    V = 70001
    target, draft, u = torch.zeros(2, 7, V, device="cuda"), torch.zeros(2, 7, V, device="cuda"), torch.zeros(2, 7, device="cuda")
    tokens, parents = torch.zeros(2, 6, dtype=torch.int32, device="cuda"), torch.tensor([[-1, -1, 0, 0, 2, 2]] * 2, dtype=torch.int32, device="cuda")
    new = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    outs = [(torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda"), new(2, 6), new(2), new(2)) for _ in "ab"]
    scratch, more = a.new_attend_scratch(ref.total, 150, weigh), binding.tree_verify_scratch(target, draft)

    def step(kv, out, lse, path, length, follows):
        kv.attend(q, starts, 150, out, lse, weigh=weigh, scratch=scratch)
        binding.tree_verify(target, tokens, parents, u, path, length, follows, draft=draft, scratch=more)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step(a, *outs[0])
    for _ in range(5):
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        x = 2 * torch.randn(target.shape, generator=g, device="cuda")
        target.copy_(torch.softmax(x, dim=2))
        draft.copy_(torch.softmax(x + torch.randn(x.shape, generator=g, device="cuda"), dim=2))
        tokens.copy_(torch.multinomial(draft[:, 0], 6, generator=g))
        u.copy_(torch.rand(u.shape, generator=g, device="cuda"))
        graph.replay()
        step(b, *outs[1])
        torch.cuda.synchronize()
        for y, z in zip(*outs):
            assert torch.equal(y, z)
        assert torch.equal(a.weights, b.weights)


def test_drafted_chains_over_pages(binding):
    """A chain of drafted tokens is appended and attended as a chunk; what is not accepted is taken back by its length."""
    import torch

    from tests.serve_reference import Paged, verify

    ref = Paged(lens=[45, 21], news=[5, 5], page_size=16, kv_heads=1, group=2, d=64, seed=6, width=5, spare=10)
    ref.table[0], ref.table[1] = torch.arange(5), torch.arange(5, 10)
    kv = ref.on_gpu(binding)
    rows = [torch.randn(10, 1, 64, generator=ref.g).to(ref.t) for _ in "kv"]
    at = torch.arange(10, dtype=torch.int32)
    kv.append(rows[0].cuda(), rows[1].cuda(), ref.starts.cuda(), at.cuda())
    ref.append(*rows, at)
    out, want = kv.attend(ref.q.cuda(), ref.starts.cuda(), 5), ref.attend()
    held(out, want["out"], want["room"])
    head = torch.randn(128, 300, generator=ref.g).cuda()
    logits = torch.cat([torch.zeros(2, 1, 300, device="cuda"), (out.float().reshape(10, 128) @ head).view(2, 5, 300)], dim=1)
    target = torch.softmax(logits, dim=2)
    draft = torch.softmax(logits + 0.3 * torch.randn(2, 6, 300, generator=ref.g).cuda(), dim=2)
    parents = torch.arange(-1, 4).int().repeat(2, 1)
    tokens = torch.stack([torch.multinomial(draft[:, i].cpu(), 1, generator=ref.g)[:, 0] for i in range(5)], dim=1).int()
    u = torch.rand(2, 6, generator=ref.g)
    new = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    path, length, follows = new(2, 5), new(2), new(2)
    binding.tree_verify(target, tokens.cuda(), parents.cuda(), u.cuda(), path, length, follows, draft=draft)
    for x, y in zip((path, length, follows), verify(target.cpu(), draft.cpu(), tokens, parents, u)):
        assert torch.equal(x.cpu(), y)
    kv.lens.sub_(5 - length)
    ref.lens -= 5 - length.cpu()
    # the next token of each, over the accepted ones alone
    ref.news, ref.starts, ref.total = [1, 1], torch.tensor([0, 1, 2], dtype=torch.int32), 2
    ref.lens += 1
    kv.lens.add_(1)
    one = [torch.randn(2, 1, 64, generator=ref.g).to(ref.t) for _ in "kv"]
    ref.q = ref.q[:2]
    kv.append(one[0].cuda(), one[1].cuda(), ref.starts.cuda(), at[:2].cuda())
    ref.append(*one, at[:2])
    want = ref.attend()
    held(kv.attend(ref.q.cuda(), ref.starts.cuda(), 1, weigh=True), want["out"], want["room"])


def test_drafted_trees_on_a_treekv_context(binding):
    """tree_attend, tree_verify, tree_commit: the path goes from one to the next on the device, captured too."""
    import torch

    from tests.serve_reference import verify

    B, H, n, d, V = 3, 2, 9, 64, 400
    kv = binding.TreeKV(32, H, d, kv_heads=H, batch=B, n_sink=2, n_recent=10)
    twin = binding.TreeKV(32, H, d, kv_heads=H, batch=B, n_sink=2, n_recent=10)
    g = torch.Generator(device="cuda").manual_seed(8)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    parents = torch.tensor([[-1, 0, 0, 1, 1, 2, -1, 6, 3]] * B, dtype=torch.int32, device="cuda")
    q, k, v = [torch.zeros(B, n, H, d, dtype=torch.bfloat16, device="cuda") for _ in "qkv"]
    head, first = rand(H * d, V) * 0.2, torch.zeros(B, 1, V, device="cuda")
    tokens, u, noise = torch.zeros(B, n, dtype=torch.int32, device="cuda"), torch.zeros(B, n + 1, device="cuda"), torch.zeros(B, n + 1, V, device="cuda")
    new = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731

    def buffers(c):
        return dict(outs=c.new_tree_outputs(n), path=new(B, n), length=new(B), follows=new(B), retained=new(B, H, 32), kept=new(B, H),
                    evicted=new(B, H, n), status=new(B), target=torch.zeros(B, n + 1, V, device="cuda"), draft=torch.zeros(B, n + 1, V, device="cuda"))

    def step(c, m):
        out, lse, scratch = m["outs"]
        c.tree_attend(q, k, v, parents, out, lse, scratch)
        logits = torch.cat([first, torch.matmul(out.view(B, n, H * d), head)], dim=1)
        m["target"].copy_(torch.softmax(logits, dim=2))
        m["draft"].copy_(torch.softmax(logits + noise, dim=2))
        binding.tree_verify(m["target"], tokens, parents, u, m["path"], m["length"], m["follows"], draft=m["draft"])
        c.tree_commit(q, k, v, parents, lse, m["path"], m["length"], m["retained"], m["kept"], m["evicted"], m["status"])

    eager, held_ = buffers(kv), buffers(twin)
    step(kv, eager)                                            # (libraries settle before the capture)
    kv.reset()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step(twin, held_)
    taken = 0
    for i in range(14):
        for x in (q, k, v):
            x.copy_(rand(*x.shape))
        tokens.copy_(torch.randint(0, V, (B, n), generator=g, device="cuda"))
        u.copy_(torch.rand(B, n + 1, generator=g, device="cuda") * 0.7)
        noise.copy_(0.3 * rand(B, n + 1, V))
        step(kv, eager)
        graph.replay()
        torch.cuda.synchronize()
        want = verify(eager["target"].cpu(), eager["draft"].cpu(), tokens.cpu(), parents.cpu(), u.cpu())
        for x, y in zip(("path", "length", "follows"), want):
            assert torch.equal(eager[x].cpu(), y), (i, x)
        for name in ("path", "length", "follows", "retained", "kept", "evicted", "status"):
            assert torch.equal(eager[name], held_[name]), (i, name)
        assert not bool(eager["status"].any())
        taken += int(eager["length"].sum())
    assert taken > 40 and torch.equal(kv.scores(), twin.scores())
