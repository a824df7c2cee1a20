"""Speculative decoding on a TreeKV cache: the operators' workloads and their plain forms.

A case is a dict of plain values; its "path" says which operator a pass goes through:

  prepare  the rows of a packed q | k | v projection become the operands of the library's calls: an RMS norm of every
           query and key head, the rotary encoding of the token's position, the values copied out of the packed rows
  attend   a tree of drafted tokens attends the cache and each token's own ancestors; nothing is changed
  commit   the accepted path of the tree enters the cache: scores, appends, evictions (Algorithm 1).  A pass hands the
           whole updated state out as a snapshot, in position order
  fork     sequences of one context are copied over sequences of another (or emptied), and the receiving context's whole
           state is handed out as a snapshot

A pass of `commit` advances the state, as it does in a user's program: the next pass on it goes on from there.

The state of a context, in the plain forms, is what a snapshot holds: per unit (sequence, KV head) the positions of the
cached tokens in ascending order, their scores S, their rows of K and V, and the counters n (tokens cached), t (tokens seen)
and idx (the eviction scope, 1 .. m).  Inputs have the distribution the configurations use: N(0, 1) plus a per-head
rank-8 part, so that a few slots carry most of the attention (fp32 storage: plain N(0, 1)).
"""
from __future__ import annotations

import math

import torch

own = False

SINKS = 4                       # the library's default layout: 4 sinks, budget/2 tree slots, the rest recent
MAX_NODES = 256                 # of a drafted tree
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One token of one sequence between two decode steps: all latency.
        dict(name="prepare_token", path="prepare", tokens=1, q_heads=32, kv_heads=32, head_dim=128, rotated=128,
             halves=False, norms=True, dtype="bf16"),
        # The drafted tokens of a batch of 16 sequences, grouped queries, half of each head rotated.
        dict(name="prepare_drafts", path="prepare", tokens=16 * 61, q_heads=32, kv_heads=8, head_dim=128, rotated=64,
             halves=True, norms=True, dtype="bf16"),
        # A 32768-token prompt before it is compressed.
        dict(name="prepare_prompt", path="prepare", tokens=32768, q_heads=32, kv_heads=8, head_dim=128, rotated=128,
             halves=True, norms=True, dtype="bf16"),
        # The tiny fp32 configuration with a small tree.
        dict(name="attend_tiny_f32", path="attend", batch=1, kv_heads=2, group=1, head_dim=64, budget=64, nodes=7,
             dtype="f32", rerank=False),
        # Interactive generation: one sequence, grouped queries, a tree of 26 drafted tokens.
        dict(name="attend_single", path="attend", batch=1, kv_heads=8, group=4, head_dim=128, budget=2048, nodes=26,
             dtype="bf16", rerank=False),
        # The headline shape (batch 8, 32 heads, 2048 slots) with 16 drafted tokens a sequence.
        dict(name="attend_batch8", path="attend", batch=8, kv_heads=32, group=1, head_dim=128, budget=2048, nodes=16,
             dtype="bf16", rerank=False),
        # Batched serving with grouped queries, the longest cache and large trees: 256 query rows a unit.
        dict(name="attend_gqa", path="attend", batch=16, kv_heads=8, group=4, head_dim=128, budget=4096, nodes=64,
             dtype="bf16", rerank=False),
        # Positions re-assigned to cache ranks, which is how the paper runs its models.
        dict(name="attend_rerank", path="attend", batch=8, kv_heads=8, group=4, head_dim=128, budget=2048, nodes=13,
             dtype="bf16", rerank=True),
        # One sequence's accepted tokens.
        dict(name="commit_single", path="commit", batch=1, kv_heads=8, group=4, head_dim=128, budget=1024, nodes=26,
             longest=5, dtype="bf16", rerank=False),
        # Eight sequences that accept between none and eight tokens each.
        dict(name="commit_batch8", path="commit", batch=8, kv_heads=32, group=1, head_dim=128, budget=2048, nodes=24,
             longest=8, dtype="bf16", rerank=False),
        # A finished sequence's place in a small batch is given to another one's state.
        dict(name="fork_one", path="fork", sources=1, batch=4, copies=1, emptied=0, kv_heads=8, head_dim=64, budget=512,
             dtype="bf16"),
        # One compressed prompt becomes the start of 15 samples of a batch of 16.
        dict(name="fork_samples", path="fork", sources=1, batch=16, copies=15, emptied=1, kv_heads=8, head_dim=128,
             budget=4096, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges: sizes over their logarithm, whatever number comes out."""
    path = rng.choice(["prepare", "prepare", "attend", "attend", "attend", "attend", "commit", "commit", "fork"])
    group = rng.choice([1, 1, 2, 4, 8])
    c = dict(path=path, kv_heads=rng.choice([2, 4, 8, 16, 32]), head_dim=rng.choice([64, 128, 128]),
             dtype=rng.choice(["bf16"] * 4 + ["f32"]))
    if path == "prepare":
        c.update(tokens=_log_int(rng, 1, 32768), q_heads=c["kv_heads"] * group, norms=rng.random() < 0.75,
                 halves=rng.random() < 0.5, rotated=rng.choice([0, 16, 32, c["head_dim"], c["head_dim"]]))
        shrink = ["tokens"]
    else:
        c.update(batch=_log_int(rng, 1, 16), budget=_log_int(rng, 64, 4096))
        shrink = ["batch", "budget"]
        if path == "fork":
            c["sources"] = _log_int(rng, 1, c["batch"])
            c["copies"] = rng.randint(1, c["batch"])
            c["emptied"] = rng.randint(0, c["batch"] - c["copies"])
        else:
            c.update(group=group, nodes=_log_int(rng, 1, 64 if path == "commit" else MAX_NODES), rerank=rng.random() < 0.25)
            if path == "commit":
                c["longest"] = _log_int(rng, 1, min(16, c["nodes"]))
    ref = [work(r) for r in listed() if r["path"] == path]
    for name in shrink:
        while c[name] > 1 and any(work(c)[n] > max(r[n] for r in ref) for n in ("bytes", "flops")):
            c[name] = (c[name] + 1) // 2
            if path == "fork" and name == "batch":
                c["sources"] = min(c["sources"], c["batch"])
                c["copies"] = min(c["copies"], c["batch"])
                c["emptied"] = min(c["emptied"], c["batch"] - c["copies"])
    return c


def _layout(budget):
    """(sinks, tree slots, recent slots) of the library's default layout."""
    recent = budget - budget // 2 - SINKS
    return SINKS, budget - SINKS - recent, recent


# ---------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call
# ---------------------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1_000_003 * (int(seed) + 1))


def _rows(g, basis, dtype, *shape):
    """[*shape, D] rows of one KV head's distribution; `basis` [Hkv, D, 8] is aligned with shape[1]."""
    x = torch.randn(*shape, basis.shape[1], generator=g, device="cuda")
    if dtype == "bf16":
        z = torch.randn(*shape, 8, generator=g, device="cuda")
        x.add_(torch.matmul(z, basis.transpose(1, 2).contiguous()[None]), alpha=4.0)
    return x.to(TYPES[dtype])


def _bases(g, case):
    shape = (case["kv_heads"], case["head_dim"], 8)
    return [torch.randn(*shape, generator=g, device="cuda") / case["head_dim"] ** 0.5 for _ in range(2)]


def _state(g, case, batch, bases):
    """Full caches in the middle of their streams; every eighth sequence (one at least, where there are four) is still
    filling.  The slots are where an eviction-in-place cache has its tokens: anywhere."""
    c, hkv, units = case["budget"], case["kv_heads"], batch * case["kv_heads"]
    sink, m, recent = _layout(c)
    rnd = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    n = torch.full((batch,), c, dtype=torch.int64, device="cuda")
    short = (rnd(batch) * (c - 1)).long() + 1
    fills = torch.arange(batch, device="cuda") % 8 == 3
    n = torch.where(fills, short, n)
    t = torch.where(fills, n, c + 1 + (rnd(batch) * 7 * c).long())
    n, t = n.repeat_interleave(hkv), t.repeat_interleave(hkv)
    free = (t - recent - sink - m).clamp(min=0)                     # positions the tree region has lost
    tree = torch.sort((rnd(units, m) * (free[:, None] + 1)).long().clamp(max=free[:, None]), dim=1).values
    tree = tree + torch.arange(m, device="cuda") + sink
    last = t[:, None] - recent + torch.arange(recent, device="cuda")
    pos = torch.cat([torch.arange(sink, device="cuda").expand(units, sink), tree, last], dim=1)
    filling = torch.arange(c, device="cuda").expand(units, c)
    pos = torch.where((n < c)[:, None], filling, pos)
    live = filling < n[:, None]
    S = torch.exp(torch.randn(units, c, generator=g, device="cuda")) * (t[:, None] - pos) * (case.get("group", 1) / c)
    s = dict(n=n.int(), t=t.int(), idx=torch.where(n < c, 1, 1 + (rnd(units) * m).long().clamp(max=m - 1)).int(),
             pos=torch.where(live, pos, -1).int(), S=torch.where(live, S, 0.0))
    for name, basis in zip("KV", bases):
        x = _rows(g, basis, case["dtype"], batch, hkv, c).reshape(units, c, case["head_dim"])
        s[name] = torch.where(live[:, :, None], x, torch.zeros((), dtype=x.dtype, device="cuda"))
    s["slots"] = torch.argsort(rnd(units, c + 1), dim=1)[:, :c].int()
    s["slots"] = torch.where((n < c)[:, None], torch.where(live, filling, -1), s["slots"]).int()
    return s


def _tree(rng, nodes, longest=0):
    """A drafted tree: parents (-1: child of the last cached token), every node after its parent.  The first `longest`
    nodes are a chain, so that a path of that length is there to be accepted."""
    parents = [i - 1 for i in range(longest)]
    for i in range(len(parents), nodes):
        # drafters go on from recent nodes rather than from any
        parents.append(-1 if i == 0 else max(-1, i - 1 - int(min(rng.expovariate(0.25), i))))
    return parents


def _buffer(kv, s):
    """The state as a snapshot of the library."""
    lay = kv.state_layout()
    buf = torch.zeros(lay.bytes, dtype=torch.uint8, device="cuda")
    header = torch.stack([s["n"], s["t"], s["idx"], torch.zeros_like(s["n"])], dim=1)
    for off, x in ((lay.header, header), (lay.positions, s["pos"]), (lay.slots, s["slots"]), (lay.S, s["S"]),
                   (lay.K, s["K"]), (lay.V, s["V"])):
        x = x.contiguous().view(torch.uint8).reshape(-1)
        buf[off:off + x.numel()] = x
    return buf


def _context(case, batch, s):
    """A context of the library that holds the state `s`, and a snapshot buffer with views of its parts."""
    from paper_2501_04987_amd import binding

    flags = binding.TREEKV_POSITION_RERANK if case.get("rerank") else 0
    kv = binding.TreeKV(case["budget"], case["kv_heads"] * case.get("group", 1), case["head_dim"],
                        kv_heads=case["kv_heads"], batch=batch, dtype=case["dtype"], flags=flags)
    buf = _buffer(kv, s)
    kv.import_state(buf)
    lay, units, c = kv.state_layout(), batch * case["kv_heads"], case["budget"]

    def view(off, dtype, *shape):
        return buf[off:off + math.prod(shape) * dtype.itemsize].view(dtype).view(*shape)

    header = view(lay.header, torch.int32, units, 4)
    snap = dict(n=header[:, 0], t=header[:, 1], idx=header[:, 2], pos=view(lay.positions, torch.int32, units, c),
                S=view(lay.S, torch.float32, units, c), K=view(lay.K, TYPES[case["dtype"]], units, c, case["head_dim"]),
                V=view(lay.V, TYPES[case["dtype"]], units, c, case["head_dim"]))
    return kv, buf, snap


def _prepare_inputs(case, seed):
    g, d = _generator(seed), case["head_dim"]
    T, H, Hkv = case["tokens"], case["q_heads"], case["kv_heads"]
    s = dict(path="prepare", case=case, eps=1e-6)
    qkv = torch.empty(T, (H + 2 * Hkv) * d, dtype=TYPES[case["dtype"]], device="cuda")
    for lo in range(0, T, 4096):                      # heads of different sizes, as projections have them
        hi = min(T, lo + 4096)
        x = torch.randn(hi - lo, H + 2 * Hkv, d, generator=g, device="cuda")
        x *= torch.exp(0.7 * torch.randn(hi - lo, H + 2 * Hkv, 1, generator=g, device="cuda"))
        qkv[lo:hi] = x.reshape(hi - lo, -1).to(qkv.dtype)
    s["qkv"] = qkv
    s["q"] = qkv[:, :H * d].unflatten(1, (H, d))
    s["k"] = qkv[:, H * d:(H + Hkv) * d].unflatten(1, (Hkv, d))
    s["v"] = qkv[:, (H + Hkv) * d:].unflatten(1, (Hkv, d))
    s["q_weight"] = s["k_weight"] = None
    if case["norms"]:
        s["q_weight"], s["k_weight"] = [(1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(qkv.dtype) for _ in "qk"]
    s["positions"] = s["inv_freq"] = None
    if case["rotated"]:
        start = int(torch.randint(0, 1 << 20, (1,), generator=g, device="cuda"))       # far into a long stream
        s["positions"] = (start + torch.arange(T, device="cuda")).int()
        i = torch.arange(case["rotated"] // 2, dtype=torch.float64, device="cuda")
        s["inv_freq"] = torch.pow(torch.tensor(500000.0, dtype=torch.float64, device="cuda"), -2.0 * i / case["rotated"])
    return s


def _tree_inputs(case, seed):
    import random

    g, rng = _generator(seed), random.Random(int(seed))
    B, hkv, G, d, n = case["batch"], case["kv_heads"], case["group"], case["head_dim"], case["nodes"]
    bases = _bases(g, case)
    s = dict(path=case["path"], case=case, state=_state(g, case, B, bases))
    s["k"] = _rows(g, bases[0], case["dtype"], B, hkv, n).transpose(1, 2).contiguous()
    s["v"] = _rows(g, bases[1], case["dtype"], B, hkv, n).transpose(1, 2).contiguous()
    q = _rows(g, bases[0], case["dtype"], B, hkv, n * G).view(B, hkv, n, G, d)
    s["q"] = q.permute(0, 2, 1, 3, 4).reshape(B, n, hkv * G, d).contiguous()
    longest = case.get("longest", 0)
    s["parents"] = torch.tensor([_tree(rng, n, longest) for _ in range(B)], dtype=torch.int32, device="cuda")
    if case["path"] == "commit":
        # the accepted path: the chain's first tokens; one sequence of a batch accepts all, the others what comes out
        lengths = [longest] + [rng.randint(0, longest) for _ in range(B - 1)]
        s["path_len"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["nodes_of_path"] = torch.arange(longest, dtype=torch.int32, device="cuda").repeat(B, 1)
        s["lse"] = _attend(s)["lse"]                   # what the attention of the same tree gave
    return s


def _fork_inputs(case, seed):
    import random

    g, rng = _generator(seed), random.Random(int(seed))
    bases = _bases(g, case)
    s = dict(path="fork", case=case, source=_state(g, case, case["sources"], bases))
    s["state"] = _state(g, case, case["batch"], bases)
    s["dst"] = rng.sample(range(case["batch"]), case["copies"] + case["emptied"])
    s["src"] = [rng.randrange(case["sources"]) for _ in range(case["copies"])] + [-1] * case["emptied"]
    hkv = case["kv_heads"]
    unit = lambda seq: torch.tensor(seq, device="cuda")[:, None] * hkv + torch.arange(hkv, device="cuda")  # noqa: E731
    s["from"] = unit([x for x in s["src"] if x >= 0]).reshape(-1)
    s["to"] = unit(s["dst"][:case["copies"]]).reshape(-1)
    if case["emptied"]:
        s["out"] = unit(s["dst"][case["copies"]:]).reshape(-1)
    return s


def _inputs(case, seed):
    return {"prepare": _prepare_inputs, "attend": _tree_inputs, "commit": _tree_inputs, "fork": _fork_inputs}[case["path"]](case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        if case["path"] == "prepare":
            s["outs"] = [torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (s["q"], s["k"], s["v"])]
        elif case["path"] == "fork":
            s["kv"], s["buf"], s["snap"] = _context(case, case["batch"], s["state"])
            s["other"] = _context(case, case["sources"], s["source"])[0]
        else:
            s["kv"], s["buf"], s["snap"] = _context(case, case["batch"], s["state"])
            B, hkv = case["batch"], case["kv_heads"]
            if case["path"] == "attend":
                s["outs"] = s["kv"].new_tree_outputs(case["nodes"])
            else:
                new = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
                s["outs"] = (new(B, hkv, case["budget"]), new(B, hkv), new(B, hkv, case["longest"]), new(B))
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    path = s["path"]
    if not own:
        return {"prepare": _prepare, "attend": _attend, "commit": _commit, "fork": _fork}[path](s)
    if path == "prepare":
        from paper_2501_04987_amd import binding

        q, k, v = binding.qkv_prepare(s["q"], s["k"], s["v"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                                      positions=s["positions"], inv_freq=s["inv_freq"], halves=s["case"]["halves"],
                                      out=s["outs"])
        return dict(q=q, k=k, v=v)
    kv = s["kv"]
    if path == "attend":
        out, lse, scratch = s["outs"]
        kv.tree_attend(s["q"], s["k"], s["v"], s["parents"], out, lse, scratch)
        return dict(out=out, lse=lse)
    if path == "commit":
        retained, n_retained, evicted, status = s["outs"]
        kv.tree_commit(s["q"], s["k"], s["v"], s["parents"], s["lse"], s["nodes_of_path"], s["path_len"], retained,
                       n_retained, evicted, status)
        kv.export_state(s["buf"])
        return dict(s["snap"], retained=retained, n_retained=n_retained, evicted=evicted, status=status)
    kv.fork(s["other"], s["src"], s["dst"])
    kv.export_state(s["buf"])
    return s["snap"]


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _rotate(x, cos, sin, halves=False):
    """Planes (2i, 2i+1), or (i, i + rotated/2), of the first 2 * cos.shape[-1] dimensions turned."""
    r = 2 * cos.shape[-1]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if halves else (x[..., 0:r:2], x[..., 1:r:2])
    y = [a * cos - b * sin, a * sin + b * cos]
    y = torch.cat(y, dim=-1) if halves else torch.stack(y, dim=-1).flatten(-2)
    return torch.cat([y, x[..., r:]], dim=-1)


def _prepare(s):
    """y = R(position) (x / sqrt(mean(x^2) + eps) * w), one head at a time; the values as they are."""
    cos = sin = None
    if s["positions"] is not None:                     # angles in 64 bits: far positions
        angle = s["positions"].double()[:, None, None] * s["inv_freq"]
        cos, sin = angle.cos().float(), angle.sin().float()

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + s["eps"]) * w.float()
        if cos is not None:
            y = _rotate(y, cos, sin, s["case"]["halves"])
        return y.to(x.dtype)

    return dict(q=one(s["q"], s["q_weight"]), k=one(s["k"], s["k_weight"]), v=s["v"].clone())


def _angles(positions, d, base=10000.0):
    """cos and sin of position * base^(-2i/d), worked out in 64 bits."""
    freq = torch.pow(torch.tensor(base, dtype=torch.float64, device="cuda"),
                     -2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    a = positions.double()[..., None] * freq
    return a.cos().float(), a.sin().float()


def _sees(parents):
    """[B, n, n]: which tokens of the tree each of them attends: itself and its ancestors."""
    B, n = parents.shape
    up = torch.eye(n, device="cuda").repeat(B, 1, 1)
    up.scatter_add_(2, parents.long().clamp(min=0)[:, :, None], (parents >= 0).float()[:, :, None])
    for _ in range(max(1, (n - 1).bit_length())):      # 1, 2, 4, .. generations
        up = (torch.bmm(up, up) > 0).float()
    return up > 0


def _operands(s):
    """Per unit, in 32 bits: queries [U, n * G, d], cached keys and values, the tree's own."""
    c = s["case"]
    B, hkv, G, d, n = c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["nodes"]
    q = s["q"].float().view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B * hkv, n * G, d)
    kn, vn = [x.float().transpose(1, 2).reshape(B * hkv, n, d) for x in (s["k"], s["v"])]
    K, V = s["state"]["K"].float(), s["state"]["V"].float()
    if c["rerank"]:
        depth = _sees(s["parents"]).sum(dim=2) - 1                                       # [B, n]
        at = (s["state"]["n"].view(B, hkv, 1) + depth[:, None]).reshape(B * hkv, n)
        K = _rotate(K, *_angles(torch.arange(K.shape[1], device="cuda")[None], d))
        kn = _rotate(kn, *_angles(at, d))
        q = _rotate(q, *_angles(at.repeat_interleave(G, dim=1), d))
    return q, K, V, kn, vn


def _attend(s):
    """o = SoftMax(q K^T / sqrt(d)) V over the cache, the ancestors and the token itself; lse = log of the softmax's sum."""
    c = s["case"]
    B, hkv, G, d, n = c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["nodes"]
    q, K, V, kn, vn = _operands(s)
    logits = torch.cat([torch.bmm(q, K.transpose(1, 2)), torch.bmm(q, kn.transpose(1, 2))], dim=2) / math.sqrt(d)
    cached = torch.arange(K.shape[1], device="cuda") < s["state"]["n"][:, None]
    tree = _sees(s["parents"]).repeat_interleave(hkv, dim=0).repeat_interleave(G, dim=1)
    seen = torch.cat([cached[:, None].expand(-1, n * G, -1), tree], dim=2)
    logits = logits.masked_fill(~seen, -math.inf)
    top = logits.amax(dim=2, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(dim=2, keepdim=True)
    out = (torch.bmm(p[:, :, :K.shape[1]], V) + torch.bmm(p[:, :, K.shape[1]:], vn)) / total
    out = out.view(B, hkv, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, hkv * G, d)
    lse = (top + torch.log(total)).view(B, hkv, n, G).permute(0, 2, 1, 3).reshape(B, n, hkv * G)
    return dict(out=out, lse=lse.contiguous())


def _commit(s):
    """The path's tokens add their probabilities to the scores; then, with the averaged scores frozen, Algorithm 1 takes them
    in one after the other: append, compare the scope's two tokens, evict the lower (the left one of equals), advance idx."""
    c, st = s["case"], s["state"]
    B, hkv, G, d, n, budget = c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["nodes"], c["budget"]
    P, units = c["longest"], c["batch"] * c["kv_heads"]
    sink, m, recent = _layout(budget)
    ar = lambda k: torch.arange(k, device="cuda")  # noqa: E731
    node = s["nodes_of_path"].long().repeat_interleave(hkv, dim=0)                        # [U, P]
    length = s["path_len"].long().repeat_interleave(hkv)
    q, K, V, kn, vn = _operands(s)
    q = q.view(units, n, G, d).gather(1, node[:, :, None, None].expand(-1, -1, G, d)).reshape(units, P * G, d)
    kn = kn.gather(1, node[:, :, None].expand(-1, -1, d))
    lse = s["lse"].view(B, n, hkv, G).permute(0, 2, 1, 3).reshape(units, n, G)
    lse = lse.gather(1, node[:, :, None].expand(-1, -1, G)).reshape(units, P * G, 1)
    cached = torch.arange(budget, device="cuda") < st["n"][:, None]
    row = ar(P).repeat_interleave(G)
    taken = row[None, :] < length[:, None]                                                # rows of accepted tokens
    p_old = torch.exp(torch.bmm(q, K.transpose(1, 2)) / math.sqrt(d) - lse)
    p_old = p_old.masked_fill(~(cached[:, None] & taken[:, :, None]), 0.0)
    p_new = torch.exp(torch.bmm(q, kn.transpose(1, 2)) / math.sqrt(d) - lse)
    p_new = p_new.masked_fill(~((row[:, None] >= ar(P)) & taken[:, :, None]), 0.0)
    S = torch.cat([st["S"] + p_old.sum(dim=1), p_new.sum(dim=1)], dim=1)                  # ids: 0 .. budget-1, then the path
    pos = torch.cat([st["pos"].long(), st["t"].long()[:, None] + ar(P)], dim=1)
    mean = S / (st["t"].long() + length)[:, None].sub(pos).float()
    count, idx = st["n"].long(), st["idx"].long()
    order = torch.cat([ar(budget).expand(units, budget), torch.full((units, 1), -1, device="cuda")], dim=1)
    evicted = torch.full((units, P), -1, device="cuda")
    k = ar(budget + 1)
    for i in range(P):                                                                    # one token after the other
        there = i < length
        appended = torch.where((k == count[:, None]) & there[:, None], budget + i, order)
        full = there & (count == budget)
        pair = appended.gather(1, (sink + idx - 1)[:, None] + ar(2))
        b = mean.gather(1, pair.clamp(min=0))
        drop = sink + idx - 1 + (b[:, 0] > b[:, 1]).long()
        gone = pos.gather(1, appended.gather(1, drop[:, None]).clamp(min=0))[:, 0]
        evicted[:, i] = torch.where(full, gone, -1)
        kept = appended.gather(1, (k + (k >= drop[:, None]).long()).clamp(max=budget))
        kept[:, budget] = -1
        order = torch.where(full[:, None], kept, appended)
        count = torch.where(there & ~full, count + 1, count)
        idx = torch.where(full, idx % m + 1, idx)
    order = order[:, :budget]
    live = ar(budget) < count[:, None]
    at = order.clamp(min=0)
    cached_row = (at < budget)[:, :, None]
    zero = torch.zeros((), dtype=st["K"].dtype, device="cuda")
    new = dict(n=count.int(), t=(st["t"] + length).int(), idx=idx.int(), pos=torch.where(live, pos.gather(1, at), -1).int(),
               S=torch.where(live, S.gather(1, at), 0.0))
    for name, x in (("K", s["k"]), ("V", s["v"])):
        path = x.transpose(1, 2).reshape(units, n, d).gather(1, node[:, :, None].expand(-1, -1, d))
        rows = torch.where(cached_row, st[name].gather(1, at.clamp(max=budget - 1)[:, :, None].expand(-1, -1, d)),
                           path.gather(1, (at - budget).clamp(min=0)[:, :, None].expand(-1, -1, d)))
        new[name] = torch.where(live[:, :, None], rows, zero)
    s["state"] = new
    return dict(new, retained=new["pos"].view(B, hkv, budget), n_retained=new["n"].view(B, hkv),
                evicted=evicted.int().view(B, hkv, P), status=torch.zeros(B, dtype=torch.int32, device="cuda"))


def _fork(s):
    st, names = s["state"], ("n", "t", "idx", "pos", "S", "K", "V")
    for name in names:
        st[name][s["to"]] = s["source"][name][s["from"]]
        if "out" in s:
            st[name][s["out"]] = {"idx": 1, "pos": -1}.get(name, 0)
    return {name: st[name].clone() for name in names}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _turn64(x, position, freq, halves=False):
    """x [.., d] in 64 bits as complex planes times exp(i * position * freq)."""
    r = 2 * freq.numel()
    planes = x[..., :r].reshape(*x.shape[:-1], 2, r // 2).transpose(-1, -2) if halves else x[..., :r].reshape(*x.shape[:-1], r // 2, 2)
    z = torch.view_as_complex(planes.contiguous()) * torch.exp(1j * (position[..., None] * freq))
    y = torch.view_as_real(z)
    y = y.transpose(-1, -2) if halves else y
    return torch.cat([y.reshape(*x.shape[:-1], r), x[..., r:]], dim=-1)


def _exact_prepare(s, case):
    got = {}
    for name in "qk":
        x, w = s[name].double(), s[name + "_weight"]
        if w is not None:
            x = x / (x.square().sum(dim=-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt() * w.double()
        if case["rotated"]:
            x = _turn64(x, s["positions"].double()[:, None], s["inv_freq"], case["halves"])
        got[name] = x
    return dict(q=got["q"], k=got["k"], v=s["v"].double())


def _exact_probabilities(s, case, unit, rows, parents, lse=None):
    """Of one unit: probabilities [rows, G, n cached + nodes] of the tree's tokens `rows`, and the log sums."""
    st, G, d = s["state"], case["group"], case["head_dim"]
    b, h = unit // case["kv_heads"], unit % case["kv_heads"]
    n = int(st["n"][unit])
    chain = []
    for i in range(case["nodes"]):
        chain.append((chain[parents[i]] if parents[i] >= 0 else set()) | {i})
    keys = torch.cat([st["K"][unit, :n], s["k"][b, :, h]]).double()
    q = s["q"][b, rows, h * G:(h + 1) * G].double()
    if case["rerank"]:
        depth = torch.tensor([len(c) - 1 for c in chain], dtype=torch.float64, device="cuda")
        at = torch.cat([torch.arange(n, dtype=torch.float64, device="cuda"), n + depth])
        freq = 10000.0 ** (-torch.arange(d // 2, dtype=torch.float64, device="cuda") * 2 / d)
        keys = _turn64(keys, at, freq)
        q = _turn64(q, (n + depth[rows])[:, None].expand(-1, G), freq)
    logits = torch.matmul(q.reshape(-1, d), keys.T.contiguous()).view(len(rows), G, -1) / math.sqrt(d)
    hidden = torch.ones(len(rows), n + case["nodes"], dtype=torch.bool)
    hidden[:, :n] = False
    for x, i in enumerate(rows):
        hidden[x, [n + j for j in chain[i]]] = False
    logits = logits.masked_fill(hidden.to(logits.device)[:, None], -math.inf)
    total = torch.logsumexp(logits, dim=2) if lse is None else lse
    return torch.exp(logits - total[:, :, None]), total


def _exact_attend(s, case):
    B, hkv, G, d, n = case["batch"], case["kv_heads"], case["group"], case["head_dim"], case["nodes"]
    out = torch.empty(B, n, hkv * G, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(B, n, hkv * G, dtype=torch.float64, device="cuda")
    parents = s["parents"].tolist()
    for unit in range(B * hkv):
        b, h = divmod(unit, hkv)
        p, total = _exact_probabilities(s, case, unit, list(range(n)), parents[b])
        values = torch.cat([s["state"]["V"][unit, :int(s["state"]["n"][unit])], s["v"][b, :, h]]).double()
        out[b, :, h * G:(h + 1) * G] = torch.matmul(p.view(n * G, -1), values).view(n, G, d)
        lse[b, :, h * G:(h + 1) * G] = total
    return dict(out=out, lse=lse)


def _exact_commit(s, case):
    """The scores and rows of every unit, from a list of its tokens that is walked as Algorithm 1 is written."""
    B, hkv, G, d, budget = case["batch"], case["kv_heads"], case["group"], case["head_dim"], case["budget"]
    sink, m, recent = _layout(budget)
    st = s["state"]
    S = torch.zeros(B * hkv, budget, dtype=torch.float64, device="cuda")
    K, V = [torch.zeros(B * hkv, budget, d, dtype=torch.float64, device="cuda") for _ in "KV"]
    parents, lengths, paths = s["parents"].tolist(), s["path_len"].tolist(), s["nodes_of_path"].tolist()
    for unit in range(B * hkv):
        b, h = divmod(unit, hkv)
        n, t, idx, path = int(st["n"][unit]), int(st["t"][unit]), int(st["idx"][unit]), paths[b][:lengths[b]]
        score = st["S"][unit, :n].double().tolist()
        if path:
            p, _ = _exact_probabilities(s, case, unit, path, parents[b], s["lse"][b, path, h * G:(h + 1) * G].double())
            p = p.sum(dim=(0, 1)).tolist()
            score = [x + y for x, y in zip(score, p[:n])] + [p[n + i] for i in path]
        where = st["pos"][unit, :n].tolist() + [t + i for i in range(len(path))]
        seen = t + len(path)
        tokens = list(range(n))
        for i in range(len(path)):
            tokens.append(n + i)
            if len(tokens) > budget:
                left, right = tokens[sink + idx - 1], tokens[sink + idx]
                of = lambda x: score[x] / (seen - where[x])  # noqa: E731
                tokens.remove(right if of(left) > of(right) else left)
                idx = idx % m + 1
        pick = torch.tensor(tokens, device="cuda")
        S[unit, :len(tokens)] = torch.tensor(score, dtype=torch.float64, device="cuda")[pick]
        K[unit, :len(tokens)] = torch.cat([st["K"][unit, :n], s["k"][b, path, h]]).double()[pick]
        V[unit, :len(tokens)] = torch.cat([st["V"][unit, :n], s["v"][b, path, h]]).double()[pick]
    return dict(S=S, K=K, V=V)


def exact(case, seed):
    s = _inputs(case, seed)
    path = case["path"]
    if path == "prepare":
        return _exact_prepare(s, case)
    if path == "attend":
        return _exact_attend(s, case)
    if path == "commit":
        return dict(_exact_commit(s, case), n=None, t=None, idx=None, pos=None, retained=None, n_retained=None, evicted=None,
                    status=None)
    got = {name: s["state"][name].double() for name in "SKV"}
    for name in "SKV":
        for x, y in zip(s["to"].tolist(), s["from"].tolist()):
            got[name][x] = s["source"][name][y].double()
        for x in s["out"].tolist() if "out" in s else []:
            got[name][x] = 0.0
    return dict(got, n=None, t=None, idx=None, pos=None)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    e, d, hkv = 2 if case["dtype"] == "bf16" else 4, case["head_dim"], case["kv_heads"]
    if case["path"] == "prepare":
        heads = case["q_heads"] + 2 * hkv
        # every head read and written once, the positions; a norm is four operations a value, a turn three
        return {"bytes": case["tokens"] * (2 * heads * d * e + 4), "flops": case["tokens"] * heads * d * 7}
    units, c = case["batch"] * hkv, case["budget"]
    if case["path"] == "fork":
        # the copied rows, scores and positions read from one context and written to the other; then the whole snapshot:
        # each unit's rows, scores and positions read and written
        row = 2 * d * e + 8
        return {"bytes": 2 * c * row * hkv * (case["copies"] + case["batch"] - case["emptied"] / 2), "flops": 0}
    G, n = case["group"], case["nodes"]
    if case["path"] == "attend":
        # the cached rows and the tree's, the queries; outputs and log sums
        per_unit = 2 * (c + n) * d * e + n * G * (d * e + 4 * d + 4)
        return {"bytes": units * per_unit + 4 * case["batch"] * n, "flops": units * 4 * G * n * d * (c + (n + 1) / 2)}
    P = case["longest"]
    # the keys read for the scores, the path's rows read and written; then the snapshot: rows, scores, positions read and
    # written (the keys have been read); the retained list
    per_unit = c * d * e + P * d * e * (4 + G) + 2 * c * 8 + 3 * c * d * e + 4 * c
    return {"bytes": units * per_unit, "flops": units * 2 * G * P * d * (c + P / 2)}
