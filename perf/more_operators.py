"""A paged cache and the verification of drafted tokens: the operators' workloads and their plain forms.

A case is a dict of plain values; its "path" says which operator a pass goes through:

  append  a chunk's keys and values go into the pages of their sequences
  attend  each sequence's chunk of new tokens attends what its pages hold, itself among it (causally); with `weigh` the
          probabilities are added to the weights of the cached tokens
  evict   sequences that have outgrown the budget keep, per KV head, the first and the last tokens and of the others those
          with the most accumulated weight; kept tokens from behind the budget move into the freed slots
  verify  which tokens of a drafted tree are accepted, from the target's and the drafter's probabilities and given uniform
          numbers, and the token that follows

The pages are [pages, kv_heads, page_size, head_dim]; `table` [batch, width] names the page of each page_size tokens of a
sequence, `lens` [batch] says how many tokens it holds, those of the chunk in hand among them; `starts` [batch + 1] are the
chunks' first rows in the packed rows of new tokens.  Weights and positions are [batch, kv_heads, width * page_size].

Keys, values and queries have the distribution the configurations use: N(0, 1) plus a per-head rank-8 part, so that a few
tokens carry most of the attention (fp32 storage: plain N(0, 1)).
"""
from __future__ import annotations

import math
import random

import torch

own = False

SINKS = 4                       # tokens at the start that eviction leaves alone; half of the budget at the end
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One new token of each sequence of a small batch: all latency.
        dict(name="append_token", path="append", batch=4, chunk=1, context=1500, page_size=16, kv_heads=8, group=4,
             head_dim=128, dtype="bf16"),
        # The chunks of four long prompts in one call.
        dict(name="append_prompt", path="append", batch=4, chunk=8192, context=0, page_size=64, kv_heads=8, group=4,
             head_dim=128, dtype="bf16"),
        # Interactive generation: one sequence, one token, grouped queries.
        dict(name="attend_token", path="attend", batch=1, chunk=1, context=2047, page_size=16, kv_heads=8, group=4,
             head_dim=128, dtype="bf16", weigh=False),
        # The tiny fp32 configuration with a chunk of an odd length; weights for a later eviction.
        dict(name="attend_tiny_f32", path="attend", batch=2, chunk=7, context=300, page_size=16, kv_heads=2, group=1,
             head_dim=64, dtype="f32", weigh=True),
        # Batched generation over long caches, with weights: every key and value once.
        dict(name="attend_decode", path="attend", batch=16, chunk=1, context=16000, page_size=32, kv_heads=8, group=4,
             head_dim=128, dtype="bf16", weigh=True),
        # A chunk of 512 tokens deep in a long prompt.
        dict(name="attend_chunk", path="attend", batch=1, chunk=512, context=32256, page_size=64, kv_heads=8, group=4,
             head_dim=128, dtype="bf16", weigh=False),
        # Whole prompts of unequal lengths, with the weights that the first eviction goes by.
        dict(name="attend_prompt", path="attend", batch=4, chunk=4000, context=0, page_size=16, kv_heads=32, group=1,
             head_dim=128, dtype="bf16", weigh=True),
        # A decode step's eviction: one token over the budget in every sequence of the headline shape.
        dict(name="evict_token", path="evict", batch=8, grown=1, budget=2048, page_size=16, kv_heads=32, group=1,
             head_dim=128, dtype="bf16"),
        # After each chunk of a prompt that is cut while it is read.
        dict(name="evict_chunk", path="evict", batch=1, grown=512, budget=1024, page_size=64, kv_heads=8, group=4,
             head_dim=128, dtype="bf16"),
        # Long prompts cut in one step, after they have been read whole.
        dict(name="evict_prompt", path="evict", batch=4, grown=28672, budget=4096, page_size=64, kv_heads=8, group=4,
             head_dim=128, dtype="bf16"),
        # Five drafted tokens in a row of one sequence.
        dict(name="verify_chain", path="verify", batch=1, nodes=5, vocab=32000, branches=1, drawn=True, dtype="f32"),
        # Trees of 26 drafted tokens for a batch, over a large vocabulary.
        dict(name="verify_trees", path="verify", batch=16, nodes=26, vocab=131072, branches=3, drawn=True, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges: sizes over their logarithm, whatever number comes out."""
    path = rng.choice(["append", "attend", "attend", "attend", "attend", "attend", "evict", "evict", "verify", "verify"])
    if path == "verify":
        c = dict(path=path, batch=_log_int(rng, 1, 32), nodes=_log_int(rng, 1, 64), vocab=_log_int(rng, 1000, 160000),
                 branches=rng.choice([1, 2, 3, 4]), drawn=rng.random() < 0.7, dtype=rng.choice(["f32", "f32", "bf16"]))
        shrink = ["nodes", "batch", "vocab"]
    else:
        c = dict(path=path, batch=_log_int(rng, 1, 16), page_size=rng.choice([16, 32, 64, 128]),
                 kv_heads=rng.choice([1, 2, 4, 8, 16, 32]), group=rng.choice([1, 1, 2, 3, 4, 7, 8]),
                 head_dim=rng.choice([64, 128, 128]), dtype=rng.choice(["bf16"] * 4 + ["f32"]))
        if path == "evict":
            c.update(budget=_log_int(rng, 64, 4096), grown=_log_int(rng, 1, 28672))
            shrink = ["grown", "batch", "budget"]
        else:
            c.update(chunk=rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 64, 4000)]),
                     context=rng.choice([0, _log_int(rng, 16, 32256), _log_int(rng, 16, 32256)]))
            if path == "attend":
                c["weigh"] = rng.random() < 0.5
            shrink = ["context", "chunk", "batch"] if path == "attend" else ["context", "batch", "chunk"]
    ref = [work(r) for r in listed() if r["path"] == path]
    size = lambda k: max(_memory(k), 1)  # noqa: E731
    most = max(size(r) for r in listed() if r["path"] == path)
    while any(work(c)[n] > max(r[n] for r in ref) for n in ("bytes", "flops")) or size(c) > most:
        big = [n for n in shrink if c[n] > (64 if n == "budget" else 1)]
        if not big:
            break
        name = max(big, key=lambda n: c[n])
        c[name] = max((c[name] + 1) // 2, 64 if name == "budget" else 1)
    return c


def _memory(case):
    """Numbers that a state holds or its plain form forms."""
    if case["path"] == "verify":
        return 2 * case["batch"] * (case["nodes"] + 1) * case["vocab"]
    cap = max(l for l, _ in _lengths(case)) + 1
    rows = case["batch"] * case["kv_heads"]
    if case["path"] == "attend":
        return rows * cap * max(case["group"] * case["chunk"], 2 * case["head_dim"])
    return rows * cap * 2 * case["head_dim"]


def _lengths(case):
    """(tokens cached, those of the chunk or the growth among them) of each sequence: unequal ones, from the case alone."""
    rng = random.Random("%d %d %d" % (case["batch"], case.get("context", case.get("budget")), case.get("chunk", case.get("grown"))))
    got = []
    for b in range(case["batch"]):
        if case["path"] == "evict":
            # the first has grown by all of it, the others by some or nothing; a single token is new in all of them
            grown = case["grown"] if b == 0 or case["grown"] == 1 else rng.randint(case["grown"] // 2, case["grown"])
            got.append((case["budget"] + grown, grown))
            continue
        # the first sequence has the full length; of five or more the fourth has no new token
        new = case["chunk"] if b == 0 or case["chunk"] == 1 else rng.randint(case["chunk"] // 2, case["chunk"])
        new = 0 if b == 3 and case["batch"] > 4 else new
        old = case["context"] if b == 0 else rng.randint(case["context"] // 4, case["context"])
        got.append((old + new, new))
    return got


# ---------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call
# ---------------------------------------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1_000_003 * (int(seed) + 1))


def _rows(g, basis, dtype, n, per_head=1):
    """[n, kv_heads * per_head, d] rows: each KV head's distribution, `per_head` draws of it side by side."""
    hkv, d, _ = basis.shape
    out = torch.empty(n, hkv * per_head, d, dtype=TYPES[dtype], device="cuda")
    for lo in range(0, n, 16384):
        hi = min(n, lo + 16384)
        x = torch.randn(hkv, (hi - lo) * per_head, d, generator=g, device="cuda")
        if dtype == "bf16":
            z = torch.randn(hkv, (hi - lo) * per_head, 8, generator=g, device="cuda")
            x.add_(torch.bmm(z, basis.transpose(1, 2).contiguous()), alpha=4.0)
        out[lo:hi] = x.view(hkv, hi - lo, per_head, d).transpose(0, 1).reshape(hi - lo, hkv * per_head, d).to(out.dtype)
    return out


def _paged(g, case, s, lens):
    """Pages handed out in any order, a few of them to nobody, and full of earlier tokens."""
    ps, hkv, d, B = case["page_size"], case["kv_heads"], case["head_dim"], case["batch"]
    need = [(l + ps - 1) // ps for l in lens]
    width = max(max(need), 1) + 1
    pages = sum(need) + 3
    free = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = free[at:at + n]
        at += n
    bases = [torch.randn(hkv, d, 8, generator=g, device="cuda") / d ** 0.5 for _ in "kv"]
    for name, basis in zip("kv", bases):
        s["cache_" + name] = _rows(g, basis, case["dtype"], pages * ps).view(pages, ps, hkv, d).transpose(1, 2).contiguous()
    s["table"], s["bases"] = table, bases
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["capacity"] = width * ps


def _chunk_inputs(case, seed):
    g = _generator(seed)
    s = dict(path=case["path"], case=case)
    lengths = _lengths(case)
    _paged(g, case, s, [l for l, _ in lengths])
    starts = [0]
    for _, n in lengths:
        starts.append(starts[-1] + n)
    s["total"], s["longest"] = starts[-1], max(n for _, n in lengths)
    s["longest_cache"] = max(l for l, _ in lengths)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    shape = (case["batch"], case["kv_heads"], s["capacity"])
    if case["path"] == "append":
        s["k"], s["v"] = [_rows(g, basis, case["dtype"], s["total"]) for basis in s["bases"]]
        far = int(torch.randint(0, 1 << 20, (1,), generator=g, device="cuda"))
        s["new_positions"] = (far + torch.arange(s["total"], device="cuda")).int()
    else:
        s["q"] = _rows(g, s["bases"][0], case["dtype"], s["total"], case["group"])
    if case.get("weigh", True):
        s["weights"] = torch.exp(torch.randn(shape, generator=g, device="cuda"))
        s["positions"] = torch.arange(s["capacity"], device="cuda").int().expand(shape).contiguous()
    return s


def _evict_inputs(case, seed):
    g = _generator(seed)
    B, hkv, budget = case["batch"], case["kv_heads"], case["budget"]
    lengths = _lengths(case)
    s = dict(path="evict", case=case, budget=budget, n_sink=SINKS, n_recent=budget // 2, longest_cache=max(l for l, _ in lengths))
    _paged(g, case, s, [l for l, _ in lengths])
    s["grown"] = torch.tensor([n for _, n in lengths], dtype=torch.int32, device="cuda")
    s["lens"] -= s["grown"]                          # as the last eviction left them; a pass adds what has come since
    C = s["capacity"]
    # slots below the budget: what earlier evictions have left there, in any order; behind them the newest tokens
    seen = budget * (1 if case["grown"] > budget else 5)
    old = torch.rand(B, hkv, seen - SINKS, generator=g, device="cuda").argsort(dim=2)[..., :budget - SINKS] + SINKS
    first = torch.arange(SINKS, device="cuda").expand(B, hkv, SINKS)
    old = torch.cat([first, old], dim=2)
    mix = torch.rand(B, hkv, budget, generator=g, device="cuda").argsort(dim=2)
    new = seen + torch.arange(C - budget, device="cuda").expand(B, hkv, C - budget)
    s["positions"] = torch.cat([old.gather(2, mix), new], dim=2).int().contiguous()
    age = (seen + s["grown"][:, None, None] - s["positions"]).clamp(min=1)
    s["weights"] = torch.exp(torch.randn(B, hkv, C, generator=g, device="cuda")) * age * (case["group"] / budget)
    return s


def _parents(rng, nodes, branches):
    """A drafted tree, level by level: up to `branches` children of each of the most recent nodes."""
    parents, at = [], -1
    while len(parents) < nodes:
        for _ in range(min(rng.randint(1, branches), nodes - len(parents))):
            parents.append(at)
        at += 1
    return parents


def _verify_inputs(case, seed):
    g, rng = _generator(seed), random.Random(int(seed))
    B, n, V = case["batch"], case["nodes"], case["vocab"]
    s = dict(path="verify", case=case)
    s["parents"] = torch.tensor([_parents(rng, n, case["branches"]) for _ in range(B)], dtype=torch.int32, device="cuda")
    s["target"] = torch.empty(B, n + 1, V, dtype=TYPES[case["dtype"]], device="cuda")
    s["draft"] = torch.empty_like(s["target"]) if case["drawn"] else None
    s["tokens"] = torch.empty(B, n, dtype=torch.int32, device="cuda")
    for b in range(B):
        # a model's logits, and a drafter that is near it
        x = 3.0 * torch.randn(n + 1, V, generator=g, device="cuda")
        y = x + 0.8 * torch.randn(n + 1, V, generator=g, device="cuda")
        s["target"][b] = torch.softmax(x, dim=1).to(s["target"].dtype)
        q = torch.softmax(y, dim=1).to(s["target"].dtype)
        row = s["parents"][b].long() + 1
        if case["drawn"]:
            s["draft"][b] = q
            up = torch.rand(n, 1, generator=g, device="cuda", dtype=torch.float64)
            cdf = q.double().cumsum(dim=1)[row]
            s["tokens"][b] = torch.searchsorted(cdf, up * cdf[:, -1:], right=True)[:, 0].clamp(max=V - 1).int()
        else:
            # the drafter's most likely tokens: the j-th child of a node has the j-th of them
            rank = torch.tensor([[p == o for o in s["parents"][b, :i].tolist()].count(True) for i, p in enumerate(s["parents"][b].tolist())])
            best = q.float().topk(min(V, n + 1), dim=1).indices[row]
            s["tokens"][b] = best.gather(1, rank.to("cuda")[:, None])[:, 0].int()
    s["uniforms"] = torch.rand(B, n + 1, generator=g, device="cuda")
    return s


def _inputs(case, seed):
    return {"append": _chunk_inputs, "attend": _chunk_inputs, "evict": _evict_inputs, "verify": _verify_inputs}[case["path"]](case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2501_04987_amd import binding

        if case["path"] == "verify":
            new = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
            s["outs"] = new(case["batch"], case["nodes"]), new(case["batch"]), new(case["batch"])
            s["scratch"] = binding.tree_verify_scratch(s["target"], s["draft"])
            return s
        pages, hkv, ps, d = s["cache_k"].shape
        kv = binding.PagedKV(pages, ps, hkv * case["group"], d, kv_heads=hkv, batch=case["batch"], table_width=s["table"].shape[1],
                             dtype=case["dtype"], tracked="weights" in s)
        kv.k.copy_(s.pop("cache_k"))
        kv.v.copy_(s.pop("cache_v"))
        kv.table.copy_(s["table"])
        kv.lens.copy_(s["lens"])
        if "weights" in s:
            kv.weights.copy_(s["weights"])
            kv.positions.copy_(s["positions"])
        s["kv"] = kv
        if case["path"] == "attend":
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
            s["scratch"] = kv.new_attend_scratch(s["total"], s["longest"], weigh=case["weigh"])
        elif case["path"] == "evict":
            s["scratch"] = kv.new_evict_scratch()
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------
def run(s):
    path = s["path"]
    if not own:
        return {"append": _append, "attend": _attend, "evict": _evict, "verify": _verify}[path](s)
    if path == "verify":
        from paper_2501_04987_amd import binding

        chosen, length, follows = s["outs"]
        binding.tree_verify(s["target"], s["tokens"], s["parents"], s["uniforms"], chosen, length, follows, draft=s["draft"],
                            scratch=s["scratch"])
        return dict(path=chosen, path_len=length, next_token=follows)
    kv = s["kv"]
    if path == "append":
        kv.append(s["k"], s["v"], s["starts"], s["new_positions"])
        return dict(k=kv.k, v=kv.v, weights=kv.weights, positions=kv.positions)
    if path == "attend":
        kv.attend(s["q"], s["starts"], s["longest"], s["out"], s["lse"], weigh=s["case"]["weigh"], scratch=s["scratch"])
        got = dict(out=s["out"], lse=s["lse"])
        return dict(got, weights=kv.weights) if s["case"]["weigh"] else got
    kv.lens.add_(s["grown"])                           # what has been appended since the last eviction
    kv.evict(s["budget"], s["n_sink"], s["n_recent"], scratch=s["scratch"])
    return dict(k=kv.k, v=kv.v, weights=kv.weights, positions=kv.positions, lens=kv.lens)


# ---------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------
def _sequence_of(s):
    """The sequence of each packed row."""
    row = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    return torch.searchsorted(s["starts"][1:].contiguous(), row, right=True)


def _append(s):
    """Row r of sequence b is token lens[b] - starts[b + 1] + r of it."""
    ps = s["case"]["page_size"]
    seq = _sequence_of(s)
    slot = (s["lens"] - s["starts"][1:])[seq] + torch.arange(s["total"], device="cuda")
    page = s["table"][seq, slot // ps].long()
    s["cache_k"][page, :, slot % ps] = s["k"]
    s["cache_v"][page, :, slot % ps] = s["v"]
    s["weights"][seq, :, slot] = 0.0
    s["positions"][seq, :, slot] = s["new_positions"][:, None]
    return dict(k=s["cache_k"], v=s["cache_v"], weights=s["weights"], positions=s["positions"])


def _gathered(s, pool, width):
    """[batch, kv_heads, width * page_size, d]: the first `width` pages of every sequence."""
    x = pool[s["table"][:, :width].long().clamp(min=0)]
    return x.transpose(1, 2).flatten(2, 3)


def _attend(s):
    """o = SoftMax(q K^T / sqrt(d)) V over the cached tokens up to the query's own; lse = log of the softmax's sum; the
    weights of a KV head add up the probabilities of its queries."""
    c, n = s["case"], s["longest"]
    B, hkv, G, d, ps = c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["page_size"]
    width = -(-s["longest_cache"] // ps)
    L = width * ps
    K, V = _gathered(s, s["cache_k"], width).float(), _gathered(s, s["cache_v"], width).float()
    new = s["starts"][1:] - s["starts"][:-1]
    i = torch.arange(n, device="cuda")
    live = i < new[:, None]                                                               # [B, n]
    row = torch.where(live, s["starts"][:-1, None] + i, s["total"]).long()
    q = torch.cat([s["q"], torch.zeros_like(s["q"][:1])])[row].float()                    # [B, n, H, d]
    q = q.view(B, n, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * G, d)
    logits = torch.matmul(q, K.transpose(2, 3).contiguous()) / math.sqrt(d)
    j = torch.arange(L, device="cuda")
    seen = j <= (s["lens"] - new)[:, None, None] + i[:, None]                             # [B, n, L]
    seen = seen & live[:, :, None] & (s["table"][:, :width] >= 0).repeat_interleave(ps, dim=1)[:, None]
    seen = seen.repeat_interleave(G, dim=1)[:, None]
    logits = logits.masked_fill(~seen, -math.inf)
    top = logits.amax(dim=3, keepdim=True)
    p = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=3, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out, lse = torch.matmul(p, V), top + torch.log(total)

    def packed(x, dtype):                                                                 # [B, hkv, n * G, w] -> rows
        x = x.view(B, hkv, n, G, -1).permute(0, 2, 1, 3, 4).reshape(B * n, hkv * G, -1)
        y = torch.zeros(s["total"] + 1, hkv * G, x.shape[2], dtype=dtype, device="cuda")
        return y.index_copy_(0, row.reshape(-1), x.to(dtype))[:-1]

    got = dict(out=packed(out, s["q"].dtype), lse=packed(lse, torch.float32)[:, :, 0])
    if c["weigh"]:
        s["weights"][:, :, :L] += p.sum(dim=2)
        got["weights"] = s["weights"]
    return got


def _evict(s):
    """The order of what is kept: the first and the last tokens, then by weight, the lower slot of equals; what is kept from
    behind the budget goes into the freed slots, both in slot order."""
    c, budget = s["case"], s["budget"]
    s["lens"] += s["grown"]
    B, hkv, d, ps = c["batch"], c["kv_heads"], c["head_dim"], c["page_size"]
    width = -(-s["longest_cache"] // ps)
    C = width * ps
    slot = torch.arange(C, device="cuda")
    there = (slot < s["lens"][:, None])[:, None]                                          # [B, 1, C]
    over = (s["lens"] > budget)[:, None, None]
    pos, w = s["positions"][:, :, :C].long(), s["weights"][:, :, :C]
    last = torch.where(there, pos, -1).amax(dim=2, keepdim=True)
    key = torch.where((pos < s["n_sink"]) | (pos > last - s["n_recent"]), math.inf, torch.where(torch.isnan(w), -math.inf, w))
    key = torch.where(there, key, -math.inf)
    order = torch.sort(key, dim=2, descending=True, stable=True).indices[:, :, :budget]
    kept = torch.zeros(B, hkv, C, dtype=torch.bool, device="cuda").scatter_(2, order, True)
    kept = torch.where(over, kept, slot < budget)
    hole, mover = ~kept[:, :, :budget], kept & (slot >= budget)
    movers = torch.sort((~mover).int(), dim=2, stable=True).indices                       # their slots first, ascending
    source = torch.where(hole, movers.gather(2, (hole.long().cumsum(dim=2) - 1).clamp(min=0)), slot[:budget])
    page = s["table"][:, :width].long().clamp(min=0)
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(hkv, device="cuda")[None, :, None]
    to_page, to_row = page[:, :-(-budget // ps)].repeat_interleave(ps, dim=1)[:, None, :budget], slot[:budget] % ps
    from_page, from_row = page[b, source // ps], source % ps
    for pool in (s["cache_k"], s["cache_v"]):
        pool[to_page, h, to_row] = pool[from_page, h, from_row]
    s["weights"][:, :, :budget] = w.gather(2, source)
    s["positions"][:, :, :budget] = s["positions"].gather(2, source)
    s["lens"].clamp_(max=budget)
    return dict(k=s["cache_k"], v=s["cache_v"], weights=s["weights"], positions=s["positions"], lens=s["lens"])


def _verify(s):
    """One walk over the nodes, which come after their parents: a child of the last accepted token is accepted with
    probability P(x) / Q(x), or P becomes what it exceeds Q by, made to sum to 1.  Without the drafter's probabilities Q is 1
    at x.  In 64 bits: whether a token is accepted or follows goes by sums next to a border."""
    c = s["case"]
    B, n, V = c["batch"], c["nodes"], c["vocab"]
    b = torch.arange(B, device="cuda")
    at, length = torch.zeros(B, dtype=torch.long, device="cuda"), torch.zeros(B, dtype=torch.long, device="cuda")
    chosen = torch.full((B, n + 1), -1, dtype=torch.int32, device="cuda")
    clean = lambda x: torch.where(x > 0, x, 0.0).double()  # noqa: E731
    P, rest = clean(s["target"][:, 0]), torch.ones(B, dtype=torch.float64, device="cuda")
    for i in range(n):
        child = s["parents"][:, i] == at - 1
        x = s["tokens"][:, i].long()
        p = P[b, x]
        if s["draft"] is not None:
            Q = clean(s["draft"][b, at])
            ok = s["uniforms"][:, i].double() * Q[b, x] < p
            left = torch.clamp(P - Q, min=0.0)
            total = left.sum(dim=1, keepdim=True)
            left = torch.where(total > 0, left / torch.where(total > 0, total, 1.0), P)
        else:
            ok = s["uniforms"][:, i].double() * rest < p
            left = P.clone()
            left[b, x] = 0.0
            rest = torch.where(child & ~ok, (rest - p).clamp(min=0.0), rest)
        yes, no = child & ok, child & ~ok
        chosen[b, torch.where(yes, length, n)] = i
        length = length + yes.long()
        at = torch.where(yes, i + 1, at)
        rest = torch.where(yes, 1.0, rest)
        P = torch.where(yes[:, None], clean(s["target"][:, i + 1]), torch.where(no[:, None], left, P))
    P = torch.where(P.sum(dim=1, keepdim=True) > 0, P, clean(s["target"][b, at]))
    cdf = P.cumsum(dim=1)
    hit = (P > 0) & (cdf > s["uniforms"][:, n:].double() * cdf[:, -1:])
    last = torch.where(P > 0, torch.arange(V, device="cuda"), -1).amax(dim=1)
    follows = torch.where(hit.any(dim=1), hit.int().argmax(dim=1), last)
    chosen = torch.where(torch.arange(n, device="cuda") < length[:, None], chosen[:, :n], -1)
    return dict(path=chosen, path_len=length.int(), next_token=follows.int())


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _tokens_of(s, pool, b, h, n):
    """Rows 0 .. n-1 of a sequence and KV head."""
    ps = pool.shape[2]
    pages = [p for p in s["table"][b].tolist() if p >= 0]
    return torch.cat([pool[p, h] for p in pages] + [pool[:0, h].reshape(0, pool.shape[3])])[:n] if ps else None


def _exact_append(s, case):
    K, V, W, P = s["cache_k"].double(), s["cache_v"].double(), s["weights"].double(), s["positions"].double()
    table, starts, lens, ps = s["table"].tolist(), s["starts"].tolist(), s["lens"].tolist(), case["page_size"]
    for b in range(case["batch"]):
        lo, hi = starts[b], starts[b + 1]
        first = lens[b] - (hi - lo)
        for at in range(first // ps, -(-lens[b] // ps)):                # page by page
            x, y = max(first, at * ps), min(lens[b], (at + 1) * ps)
            rows = slice(lo + x - first, lo + y - first)
            K[table[b][at], :, x - at * ps:y - at * ps] = s["k"][rows].double().transpose(0, 1)
            V[table[b][at], :, x - at * ps:y - at * ps] = s["v"][rows].double().transpose(0, 1)
        W[b, :, first:lens[b]] = 0.0
        P[b, :, first:lens[b]] = s["new_positions"][lo:hi].double()
    return dict(k=K, v=V, weights=W, positions=P.int())


def _exact_attend(s, case):
    G, d = case["group"], case["head_dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    W = s["weights"].double() if case["weigh"] else None
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    for b in range(case["batch"]):
        lo, hi, n = starts[b], starts[b + 1], starts[b + 1] - starts[b]
        if not n:
            continue
        hidden = torch.ones(n, lens[b], dtype=torch.bool, device="cuda").triu(lens[b] - n + 1)[:, None]
        for h in range(case["kv_heads"]):
            keys, values = [_tokens_of(s, s[x], b, h, lens[b]).double() for x in ("cache_k", "cache_v")]
            q = s["q"][lo:hi, h * G:(h + 1) * G].double().reshape(n * G, d)
            x = (torch.matmul(q, keys.T.contiguous()) / math.sqrt(d)).view(n, G, -1).masked_fill(hidden, -math.inf)
            lse[lo:hi, h * G:(h + 1) * G] = torch.logsumexp(x, dim=2)
            p = torch.softmax(x, dim=2)
            out[lo:hi, h * G:(h + 1) * G] = torch.matmul(p.view(n * G, -1), values).view(n, G, d)
            if W is not None:
                W[b, h, :lens[b]] += p.sum(dim=(0, 1))
    got = dict(out=out, lse=lse)
    return dict(got, weights=W) if W is not None else got


def _exact_evict(s, case):
    """Unit by unit, from a list of its tokens."""
    budget, ps = s["budget"], case["page_size"]
    K, V, W, P = s["cache_k"].double(), s["cache_v"].double(), s["weights"].double(), s["positions"].clone()
    weights, positions, table = s["weights"].cpu().tolist(), s["positions"].cpu().tolist(), s["table"].tolist()
    lens = (s["lens"] + s["grown"]).tolist()
    for b in range(case["batch"]):
        if lens[b] <= budget:
            continue
        for h in range(case["kv_heads"]):
            w, pos = weights[b][h][:lens[b]], positions[b][h][:lens[b]]
            newest = max(pos)
            safe = [x < s["n_sink"] or x > newest - s["n_recent"] for x in pos]
            order = sorted(range(lens[b]), key=lambda i: (not safe[i], 0.0 if safe[i] else -w[i], i))
            keep = set(order[:budget])
            to = [i for i in range(budget) if i not in keep]
            come = [i for i in range(budget, lens[b]) if i in keep]
            if not to:
                continue
            ti, ci, row = torch.tensor(to), torch.tensor(come), torch.tensor(table[b])
            K[row[ti // ps], h, ti % ps] = s["cache_k"][row[ci // ps], h, ci % ps].double()
            V[row[ti // ps], h, ti % ps] = s["cache_v"][row[ci // ps], h, ci % ps].double()
            W[b, h, ti] = s["weights"][b, h, ci].double()
            P[b, h, ti] = s["positions"][b, h, ci]
    return dict(k=K, v=V, weights=W, positions=P, lens=torch.tensor([min(x, budget) for x in lens], dtype=torch.int32))


def _exact_verify(s, case):
    """Sequence by sequence, each along its own path."""
    n, V = case["nodes"], case["vocab"]
    paths, lengths, follows = [], [], []
    positive = lambda x: x.double().clamp(min=0.0)  # noqa: E731
    for b in range(case["batch"]):
        parents, tokens, u = s["parents"][b].tolist(), s["tokens"][b].tolist(), s["uniforms"][b].double().tolist()
        path, at, moved = [], -1, True
        while moved:
            moved = False
            target = positive(s["target"][b, at + 1])
            P, gone = target.clone(), 0.0
            for i in [i for i in range(n) if parents[i] == at]:
                x = tokens[i]
                if s["draft"] is not None:
                    Q = positive(s["draft"][b, at + 1])
                    if u[i] * float(Q[x]) < float(P[x]):
                        path, at, moved = path + [i], i, True
                        break
                    left = (P - Q).clamp(min=0.0)
                    if float(left.sum()) > 0.0:
                        P = left / left.sum()
                else:
                    if u[i] * max(0.0, 1.0 - gone) < float(P[x]):
                        path, at, moved = path + [i], i, True
                        break
                    gone += float(P[x])
                    P[x] = 0.0
        if float(P.sum()) == 0.0:
            P = target
        cdf = P.cumsum(dim=0)
        one = torch.nonzero((P > 0) & (cdf > u[n] * cdf[-1]))
        follows.append(int(one[0]) if len(one) else int(torch.nonzero(P > 0)[-1]) if bool((P > 0).any()) else -1)
        paths.append(path + [-1] * (n - len(path)))
        lengths.append(len(path))
    new = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return dict(path=new(paths), path_len=new(lengths), next_token=new(follows))


def exact(case, seed):
    s = _inputs(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict, "verify": _exact_verify}[case["path"]](s, case)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["path"] == "verify":
        # the rows that the token after the path is drawn from, and the same once more where a draw has been refused
        rows = 2 if case["drawn"] else 1
        return {"bytes": case["batch"] * (rows * case["vocab"] * e + 16 * case["nodes"]), "flops": case["batch"] * rows * case["vocab"]}
    d, hkv, G = case["head_dim"], case["kv_heads"], case["group"]
    lengths = _lengths(case)
    if case["path"] == "append":
        # every row read and written once, a weight and a position written
        return {"bytes": sum(n for _, n in lengths) * (hkv * (4 * d * e + 8) + 4), "flops": 0}
    if case["path"] == "attend":
        # the cached rows, the queries and what comes out; two products per query and token it sees
        size = flops = 0
        for l, n in lengths:
            if n:
                size += hkv * l * (2 * d * e + (8 if case["weigh"] else 0)) + n * G * hkv * (2 * d * e + 4)
                flops += 4 * d * G * hkv * n * (l - (n - 1) / 2)
        return {"bytes": size, "flops": flops}
    # every weight and position read; rows that are kept behind the budget read and written, with weight and position
    size, budget = 0, case["budget"]
    recent = budget // 2
    for l, grown in lengths:
        new = min(grown, recent)
        moved = new + (grown - new) * max(0, budget - recent - SINKS) / max(1, l - recent - SINKS)
        size += hkv * (l * 8 + moved * (4 * d * e + 16))
    return {"bytes": size, "flops": 0}
