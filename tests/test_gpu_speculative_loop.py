"""GPU: the calls of speculative decoding in a row, as a serving loop makes them.  A prompt's projection is prepared and fed, its
sequence forked into a batch, and rounds of prepare / verify / commit, one captured graph for all of them, run beside a context
for each sequence that is fed the accepted tokens as chunks."""
import random

import pytest

pytestmark = pytest.mark.gpu
BATCH, HQ, HKV, D, NODES, LONGEST = 3, 8, 2, 64, 11, 5


@pytest.fixture(scope="module")
def binding():
    import torch

    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2501_04987_amd import binding as b

    b.load()
    return b


def packed(seed, tokens, dtype):
    import torch

    return torch.randn(tokens, (HQ + 2 * HKV) * D, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


@pytest.mark.parametrize("flags", [0, 8])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_serving_loop(binding, dt, flags):
    import torch

    dtype = torch.bfloat16 if dt == "bf16" else torch.float32
    new = lambda batch: binding.TreeKV(80, HQ, D, kv_heads=HKV, batch=batch, dtype=dt, flags=flags, n_sink=2, n_recent=30)  # noqa: E731
    weight = (1 + 0.2 * torch.randn(D, generator=torch.Generator().manual_seed(0))).to(dtype).cuda()
    freq = binding.rope_frequencies(D)

    def prepare(rows, positions, out=None):
        q, k, v = [x.unflatten(1, (-1, D)) for x in rows.split([HQ * D, HKV * D, HKV * D], dim=1)]
        turn = dict(to_planes=True) if flags else dict(positions=positions, inv_freq=freq)   # (a context of ranks turns them itself)
        return binding.qkv_prepare(q, k, v, q_weight=weight, k_weight=weight, halves=True, out=out, **turn)

    prompt, kv = new(1), new(BATCH)
    at = 0
    for seed, n in ((1, 64), (2, 61)):
        x = prepare(packed(seed, n, dtype), torch.arange(at, at + n, device="cuda").int())
        o, r, nr, ev = prompt.new_outputs(n)
        prompt.prefill_chunk(*[y[None] for y in x], n, o, r, nr, ev)
        at += n
    kv.fork(prompt, [0] * BATCH, list(range(BATCH)))
    twins = [new(1) for _ in range(BATCH)]
    for twin in twins:
        twin.fork(prompt, [0], [0])

    # what a round reads and writes, where a graph finds it
    rows, positions = packed(0, BATCH * NODES, dtype), torch.zeros(BATCH * NODES, dtype=torch.int32, device="cuda")
    parents, path = [torch.zeros(BATCH, n, dtype=torch.int32, device="cuda") for n in (NODES, LONGEST)]
    lengths, status = [torch.zeros(BATCH, dtype=torch.int32, device="cuda") for _ in range(2)]
    heads = [torch.empty(BATCH * NODES, h, D, dtype=dtype, device="cuda") for h in (HQ, HKV, HKV)]
    out, lse, scratch = kv.new_tree_outputs(NODES)
    retained, nret = kv.new_outputs()[1:3]
    evicted = torch.empty(BATCH, HKV, LONGEST, dtype=torch.int32, device="cuda")

    def round_of():
        prepare(rows, positions, heads)
        q, k, v = [x.view(BATCH, NODES, -1, D) for x in heads]
        kv.tree_attend(q, k, v, parents, out, lse, scratch)
        kv.tree_commit(q, k, v, parents, lse, path, lengths, retained, nret, evicted, status)

    rng, seen, graph = random.Random(3), [at] * BATCH, None
    for rnd in range(12):
        drafted, taken, where = [], [], []
        for b in range(BATCH):
            p = [rng.randint(-1, i - 1) if i else -1 for i in range(NODES)]
            nodes = sorted(rng.sample(range(NODES), rng.randint(0, LONGEST)))
            for x, node in enumerate(nodes):
                p[node] = nodes[x - 1] if x else -1
            depth = []
            for x in p:
                depth.append(depth[x] + 1 if x >= 0 else 0)
            drafted.append(p), taken.append(nodes), where.extend(seen[b] + x for x in depth)
        rows.copy_(packed(100 + rnd, BATCH * NODES, dtype))
        positions.copy_(torch.tensor(where, dtype=torch.int32))
        parents.copy_(torch.tensor(drafted, dtype=torch.int32))
        path.copy_(torch.tensor([x + [0] * (LONGEST - len(x)) for x in taken], dtype=torch.int32))
        lengths.copy_(torch.tensor([len(x) for x in taken], dtype=torch.int32))
        if rnd < 2:
            round_of()
        else:
            if graph is None:
                torch.cuda.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    round_of()
            graph.replay()
        assert status.tolist() == [0] * BATCH
        for b, (twin, nodes) in enumerate(zip(twins, taken)):
            L = len(nodes)
            if L:
                mine = rows.view(BATCH, NODES, -1)[b, nodes]
                x = prepare(mine, torch.arange(seen[b], seen[b] + L, device="cuda").int())
                o, r, nr, ev = twin.new_outputs(L)
                twin.prefill_chunk(*[y[None] for y in x], L, o, r, nr, ev)
                assert torch.equal(ev[0], evicted[b, :, :L]) and torch.equal(r[0], retained[b]) and torch.equal(nr[0], nret[b])
                # chunks cut P in two bf16 parts (2^-17 of values below 8) and, re-assigned, turned operands too
                assert torch.allclose(out[b, nodes], o[0], rtol=0, atol=2e-4 if dt == "bf16" else 1e-5)
                seen[b] += L
    assert min(seen) > at
    for b, twin in enumerate(twins):
        for x, y in zip(kv.gather_kv(), twin.gather_kv()):
            assert torch.equal(x[b], y[0])
