"""The paged cache and the verification of drafts in 64 bits, on the CPU, token by token as include/treekv.h defines them."""
import math

import torch


class Paged:
    """A paged cache with host copies of everything, and the same on the GPU as a binding.PagedKV."""

    def __init__(self, *, lens, news, page_size, kv_heads, group, d, dtype="bf16", width=None, seed=0, tracked=True, spare=2, scale=0.0):
        g = torch.Generator().manual_seed(seed)
        self.t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.dtype, self.ps, self.hkv, self.G, self.d, self.scale = dtype, page_size, kv_heads, group, d, scale or d ** -0.5
        self.softmax_scale = scale
        self.B, self.news = len(lens), list(news)
        need = [-(-max(n, 0) // page_size) for n in lens]
        self.width = width or max(max(need), 1) + 1
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g).tolist()
        self.table = torch.full((self.B, self.width), -1, dtype=torch.int32)
        for b, n in enumerate(need):
            for i in range(min(n, self.width)):
                self.table[b, i] = order.pop()
        self.lens = torch.tensor(lens, dtype=torch.int32)
        shape = (self.pages, kv_heads, page_size, d)
        self.k, self.v = [torch.randn(shape, generator=g).mul(1.5).to(self.t) for _ in "kv"]
        self.weights = torch.rand(self.B, kv_heads, self.width * page_size, generator=g) if tracked else None
        self.positions = torch.arange(self.width * page_size).int().expand(self.B, kv_heads, -1).contiguous() if tracked else None
        starts = [0]
        for n in self.news:
            starts.append(starts[-1] + n)
        self.starts, self.total = torch.tensor(starts, dtype=torch.int32), starts[-1]
        self.q = torch.randn(self.total, kv_heads * group, d, generator=g).mul(1.5).to(self.t)
        self.g = g

    def on_gpu(self, binding):
        kv = binding.PagedKV(self.pages, self.ps, self.hkv * self.G, self.d, kv_heads=self.hkv, batch=self.B, table_width=self.width,
                             dtype=self.dtype, tracked=self.weights is not None, softmax_scale=self.softmax_scale)
        for name in ("k", "v", "table", "lens", "weights", "positions"):
            if getattr(self, name) is not None:
                getattr(kv, name).copy_(getattr(self, name))
        return kv

    def row(self, b, slot):
        """(page, row) of a slot, page -1 where it has been given up."""
        page = int(self.table[b, slot // self.ps])
        return (page if 0 <= page < self.pages else -1), slot % self.ps

    def tokens(self, pool, b, h, n):
        """[n, d] in 64 bits and which of them are there."""
        where = [self.row(b, s) for s in range(n)]
        x = torch.zeros(n, self.d, dtype=torch.float64)
        there = torch.tensor([p >= 0 for p, _ in where], dtype=torch.bool)
        for s, (p, r) in enumerate(where):
            if p >= 0:
                x[s] = pool[p, h, r].double()
        return x, there

    def attend(self, q=None, sequences=None):
        """out, lse, what each weight gains, and the bounds their errors are held to."""
        q = self.q if q is None else q
        H, n64 = self.hkv * self.G, torch.float64
        out, room = [torch.zeros(self.total, H, self.d, dtype=n64) for _ in "or"]
        lse, lse_room = torch.full((self.total, H), -math.inf, dtype=n64), torch.zeros(self.total, H, dtype=n64)
        gain, gain_room = [torch.zeros(self.B, self.hkv, self.width * self.ps, dtype=n64) for _ in "gr"]
        # bf16: each probability is rounded once on its way into the second product, and the result once
        half = torch.finfo(self.t).eps / 2 if self.t == torch.bfloat16 else 0.0
        tiny = 2.0 ** -24
        for b in range(self.B) if sequences is None else sequences:
            lo, n, L = int(self.starts[b]), self.news[b], int(self.lens[b])
            for h in range(self.hkv if n else 0):
                K, there = self.tokens(self.k, b, h, L)
                V, _ = self.tokens(self.v, b, h, L)
                for i in range(n):
                    see = torch.arange(L) <= L - n + i
                    see &= there
                    if not bool(see.any()):
                        continue
                    k, v = K[see], V[see]
                    x = q[lo + i, h * self.G:(h + 1) * self.G].double()
                    s = x @ k.T * self.scale
                    # a logit is a sum of d products, scaled, in fp32; its error is that of its exponential and of the sums
                    d_logit = (self.d + 8) * tiny * ((x.abs() @ k.abs().T).amax(dim=1) * abs(self.scale) + s.abs().amax(dim=1))
                    total = torch.logsumexp(s, dim=1)
                    p = torch.exp(s - total[:, None])
                    # exponentials and sums of up to L terms in fp32, the reference's changes and the merges among them
                    eps = 2 * d_logit + (L + 64) * tiny
                    at = slice(h * self.G, (h + 1) * self.G)
                    out[lo + i, at], lse[lo + i, at] = p @ v, total
                    size = p @ v.abs()
                    room[lo + i, at] = (half + eps[:, None]) * size * (1 + half) + half * out[lo + i, at].abs() + 1e-30
                    lse_room[lo + i, at] = d_logit + (L + 64) * tiny + 2 * tiny * total.abs()
                    full = torch.zeros(self.G, L, dtype=n64)
                    full[:, see] = p
                    gain[b, h, :L] += full.sum(dim=0)
                    # the weights' exponential takes the rounded log sum; then a sum over the rows
                    gain_room[b, h, :L] += (full * (2 * eps + 4 * tiny * (total.abs() + s.abs().amax(dim=1)) + (n * self.G + 8) * tiny)[:, None]).sum(dim=0)
        return dict(out=out, room=room, lse=lse, lse_room=lse_room, gain=gain, gain_room=gain_room)

    def append(self, k, v, positions=None):
        for b in range(self.B):
            lo, n, L = int(self.starts[b]), self.news[b], int(self.lens[b])
            for i in range(n):
                slot = L - n + i
                page, r = self.row(b, slot)
                if page >= 0:
                    self.k[page, :, r], self.v[page, :, r] = k[lo + i], v[lo + i]
                if self.weights is not None:
                    self.weights[b, :, slot] = 0.0
                    self.positions[b, :, slot] = positions[lo + i]

    def evict(self, budget, n_sink, n_recent):
        for b in range(self.B):
            L = int(self.lens[b])
            if L <= budget or L > self.width * self.ps or any(self.row(b, s)[0] < 0 for s in range(L)):
                continue
            for h in range(self.hkv):
                w, pos = self.weights[b, h, :L].tolist(), self.positions[b, h, :L].tolist()
                last = max(pos)
                safe = [x < n_sink or x > last - n_recent for x in pos]
                rank = lambda i: (not safe[i], 0.0 if safe[i] else math.inf if math.isnan(w[i]) else -w[i], i)  # noqa: E731
                keep = set(sorted(range(L), key=rank)[:budget])
                to = [i for i in range(budget) if i not in keep]
                come = [i for i in range(budget, L) if i in keep]
                assert len(to) == len(come)
                for x, y in zip(to, come):
                    (tp, tr), (cp, cr) = self.row(b, x), self.row(b, y)
                    self.k[tp, h, tr], self.v[tp, h, tr] = self.k[cp, h, cr], self.v[cp, h, cr]
                    self.weights[b, h, x], self.positions[b, h, x] = self.weights[b, h, y], self.positions[b, h, y]
            self.lens[b] = budget


def verify(target, draft, tokens, parents, uniforms):
    """-> path [batch, n], path_len, next_token: each step written as the rule says it, with distributions in 64 bits."""
    B, rows, V = target.shape
    n = rows - 1
    positive = lambda x: torch.where(x > 0, x, torch.zeros((), dtype=x.dtype)).double()  # noqa: E731
    paths, lengths, follows = [], [], []
    for b in range(B):
        path, at, moved = [], -1, True
        while moved:
            moved, refused = False, 0.0
            P = positive(target[b, at + 1])
            for i in range(at + 1, n):
                x = int(tokens[b, i])
                if int(parents[b, i]) != at or not 0 <= x < V:
                    continue
                u = float(uniforms[b, i])
                if draft is not None:
                    Q = positive(draft[b, at + 1])
                    if u * float(Q[x]) < float(P[x]):
                        moved = True
                    else:
                        left = (P - Q).clamp(min=0)
                        if float(left.sum()) > 0:
                            P = left / left.sum()
                elif u * max(0.0, 1.0 - refused) < float(P[x]):
                    moved = True
                else:
                    refused += float(P[x])
                    P[x] = 0.0
                if moved:
                    path, at = path + [i], i
                    break
        if not float(P.sum()) > 0:
            P = positive(target[b, at + 1])
        cdf, u = P.cumsum(0), float(uniforms[b, n])
        hit = torch.nonzero((P > 0) & (cdf > u * cdf[-1]))[:, 0]
        some = torch.nonzero(P > 0)[:, 0]
        follows.append(int(hit[0]) if len(hit) else int(some[-1]) if len(some) else -1)
        paths.append(path + [-1] * (n - len(path)))
        lengths.append(len(path))
    return [torch.tensor(x, dtype=torch.int32) for x in (paths, lengths, follows)]
