"""Plain 64-bit form of a drafted tree's attention and of a path's commit, one (sequence, KV head) at a time, on the CPU.

Written from the definitions: a token attends the cache, its ancestors and itself; the path's tokens add their
probabilities to the scores; Algorithm 1's loop then takes them in with the averaged scores frozen."""
import math

import torch


def part(buf, off, dtype, *shape):
    return buf[off:off + math.prod(shape) * dtype.itemsize].view(dtype).view(*shape)


def state(kv):
    """The context's state on the host: lists per unit (sequence * kv_heads + head) of dicts."""
    c, lay, buf = kv.cfg, kv.state_layout(), kv.export_state().cpu()
    units, dt = c.batch * c.kv_heads, torch.bfloat16 if c.dtype == 0 else torch.float32
    header = part(buf, lay.header, torch.int32, units, 4)
    pos = part(buf, lay.positions, torch.int32, units, c.budget)
    S = part(buf, lay.S, torch.float32, units, c.budget)
    K, V = [part(buf, off, dt, units, c.budget, c.head_dim) for off in (lay.K, lay.V)]
    found = []
    for u in range(units):
        n, t, idx, _ = header[u].tolist()
        found.append(dict(n=n, t=t, idx=idx, pos=pos[u, :n].tolist(), S=S[u, :n].double(), K=K[u, :n].double(), V=V[u, :n].double()))
    return found


def chains(parents):
    """Per node the list of nodes it attends, ascending; None for an absent one."""
    got = []
    for i, p in enumerate(parents):
        if p == -1:
            got.append([i])
        elif 0 <= p < i and got[p] is not None:
            got.append(got[p] + [i])
        else:
            got.append(None)
    return got


def turn(x, at, base):
    d = x.shape[-1]
    angle = at[..., None] * base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], d // 2, 2).contiguous()) * torch.polar(torch.ones_like(angle), angle)
    return torch.view_as_real(z).reshape(x.shape)


def attend_unit(kv, st, q, k, v, parents):
    """q [n, G, d], k and v [n, d], all float64 -> out [n, G, d], lse [n, G], bound [n, G, d] (what fp32 may be off by), and
    per present node its probabilities [G, cached + chain]."""
    c = kv.cfg
    n, G, d = q.shape
    out, lse, bound = torch.zeros(n, G, d, dtype=torch.float64), torch.full((n, G), -math.inf, dtype=torch.float64), torch.zeros(n, G, d, dtype=torch.float64)
    probs, lse_bound = [None] * n, torch.zeros(n, G, dtype=torch.float64)
    rerank = bool(c.flags & 8)
    for i, chain in enumerate(chains(parents)):
        if chain is None:
            continue
        keys, values, query = torch.cat([st["K"], k[chain]]), torch.cat([st["V"], v[chain]]), q[i]
        if rerank:
            keys = turn(keys, torch.arange(len(keys), dtype=torch.float64), c.rope_base)
            query = turn(query, torch.full((G,), float(len(keys) - 1), dtype=torch.float64), c.rope_base)
        logits = query @ keys.T * c.softmax_scale
        lse[i] = torch.logsumexp(logits, dim=1)
        p = torch.exp(logits - lse[i][:, None])
        probs[i] = p
        out[i] = p @ values
        # A logit in fp32: d products added, the scale, and for turned operands three more roundings each, every one of them
        # at most 2^-24 of the sum of the products' sizes; the exponent of the probability is off by that, for the token and
        # for the sum, and its own rounding (a few 2^-24) and the sums over the columns (one rounding each) come on top.
        size = query.abs() @ keys.abs().T * c.softmax_scale
        step = (d + 4 + (12 if rerank else 0)) * 2.0 ** -24 * size.max(dim=1).values + 2.0 ** -24 * lse[i].abs() * 4
        each = 2 * step + (len(keys) + 16) * 2.0 ** -24
        bound[i] = torch.expm1(each)[:, None] * (p @ values.abs())
        lse_bound[i] = torch.expm1(each)
    return out, lse, bound, lse_bound, probs


def commit_unit(kv, st, q, k, v, parents, path):
    """-> the state after the path's tokens, and the positions evicted as each came in (-1: none)."""
    c = kv.cfg
    m = c.budget - c.n_sink - c.n_recent
    n, t, idx = st["n"], st["t"], st["idx"]
    score = st["S"].tolist() + [0.0] * len(path)
    if path:
        probs = attend_unit(kv, st, q, k, v, parents)[4]
        for x, node in enumerate(path):
            for j, p in enumerate(probs[node].sum(dim=0).tolist()):
                score[j] += p                         # cached tokens, then the chain: the path's tokens so far
    where = st["pos"] + [t + i for i in range(len(path))]
    seen = t + len(path)
    mean = [s if c.flags & 4 else s / (seen - w) for s, w in zip(score, where)]
    tokens, evicted, margin = list(range(n)), [], math.inf
    for i in range(len(path)):
        tokens.append(n + i)
        if len(tokens) <= c.budget:
            evicted.append(-1)
            continue
        left, right = tokens[c.n_sink + idx - 1], tokens[c.n_sink + idx]
        if not c.flags & 1 and mean[left] != mean[right]:
            margin = min(margin, abs(mean[left] - mean[right]) / max(mean[left], mean[right]))
        gone = right if (c.flags & 1) or mean[left] > mean[right] else left
        tokens.remove(gone)
        evicted.append(where[gone])
        idx = idx % m + 1
    K, V = torch.cat([st["K"], k[path]]), torch.cat([st["V"], v[path]])
    new = dict(n=len(tokens), t=seen, idx=idx, pos=[where[x] for x in tokens], S=torch.tensor([score[x] for x in tokens], dtype=torch.float64),
               K=K[tokens], V=V[tokens])
    return new, evicted, margin
