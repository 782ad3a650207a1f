"""Plain implementations in 64 bits of what a sampled, drafted turn over a bounded cache needs, one row or sequence at a time."""
import numpy as np
import torch


def cache_of(B, dtype, *, layers=1, page, kv_heads, head_dim, lens, room=None, spare=3, seed=0, values=1.0):
    """A PagedCache whose sequences 0.. have the given lengths, their pages in random order; every value of the pool is drawn."""
    rng = np.random.default_rng(seed)
    room = lens if room is None else room
    pages = [max(0, -(-r // page)) for r in room]
    total = sum(pages) + spare
    c = B.PagedCache(layers=layers, pages=total, page_size=page, kv_heads=kv_heads, head_dim=head_dim, max_seqs=len(lens), max_pages=max(1, max(pages)), dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for x in (c.k, c.v):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda") * values)
    ids, at = rng.permutation(total), 0
    table, ref = np.full((len(lens), max(1, max(pages))), -1, np.int32), np.zeros(total, np.int32)
    for s, n in enumerate(lens):
        m = -(-n // page)
        table[s, :m] = ids[at:at + m]
        ref[ids[at:at + m]] = 1
        at += pages[s]
    c.page_table.copy_(torch.tensor(table))
    c.page_ref.copy_(torch.tensor(ref))
    c.seq_len.copy_(torch.tensor(np.asarray(lens, np.int32)))
    return c


def rows_of(pool, table, page, length):
    """Rows [length, kv_heads, head_dim] of one layer's pool [pages, kv_heads, page, head_dim] that a page table row names."""
    out = [pool[int(table[p // page]), :, p % page] for p in range(length)]
    return torch.stack(out) if out else pool.new_zeros((0, pool.shape[1], pool.shape[3]))


def rotate(x, weight, eps, position, inv_freq, rot, neighbours):
    """x [T, heads, d] float64 on the host.  Returns the result and, element by element, the size that its rounding errors go by."""
    x = x.double().cpu().numpy()
    T, heads, d = x.shape
    y = x.copy()
    if weight is not None:
        y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight.double().cpu().numpy()
    out, size = y.copy(), np.abs(y)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
        angle = np.asarray(position, np.float64)[:, None] * float(inv_freq[i])
        out[..., a] = y[..., a] * np.cos(angle) - y[..., b] * np.sin(angle)
        out[..., b] = y[..., a] * np.sin(angle) + y[..., b] * np.cos(angle)
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size


def target(x, temperature):
    """Probabilities of a row of logits (float64); zeros where nothing is eligible."""
    ok = np.isfinite(x)
    p = np.zeros(len(x))
    if not ok.any():
        return p
    y = np.where(ok, x, -np.inf)
    if not (temperature > 0 and np.isfinite(temperature)):
        p[int(np.argmax(y))] = 1.0
        return p
    w = np.exp((y - y.max()) / float(temperature))
    return w / w.sum()


def verify(logits, tokens, cu, u, u_next, parent=None, near=None, temperature=None, most=None):
    """Rows that the walk takes and the next token, per sequence."""
    keep, nxt = [], []
    for i in range(len(cu) - 1):
        a, n = int(cu[i]), int(cu[i + 1] - cu[i])
        if n == 0:
            keep.append([])
            nxt.append(-1)
            continue
        t = 1.0 if temperature is None else float(temperature[i])
        V = logits.shape[1]
        path = [0]
        p = target(logits[a], t)
        r = p.copy()
        while len(path) < (most or n + 1):
            for j in range(path[-1] + 1, n):
                if (j - 1 if parent is None else int(parent[a + j])) != path[-1] or not 0 <= tokens[a + j] < V:
                    continue
                x, R = int(tokens[a + j]), r.sum() if r is not p else 1.0
                if near is None:
                    q = np.zeros(V)
                    q[x] = 1.0
                else:
                    q = near[a + path[-1]].astype(np.float64)
                    q = np.where(np.isfinite(q) & (q > 0), q, 0.0)
                if float(u[a + j]) * q[x] * R < r[x]:
                    path.append(j)
                    break
                r = np.maximum(r - q * R, 0)
                if not r.sum() > 0:
                    r = p.copy()
            else:
                break
            p = target(logits[a + path[-1]], t)
            r = p.copy()
        total = np.cumsum(r)
        keep.append(path)
        nxt.append(int(np.searchsorted(total, float(u_next[i]) * total[-1], side="right")) if total[-1] > 0 else -1)
        if nxt[-1] == V:                       # u_next rounds up to all of it
            nxt[-1] = int(np.flatnonzero(r > 0)[-1])
    return keep, nxt


def weigh(q, lse, k, scale, rows, base):
    """Weights [len(k)] that the counted packed rows add (float64), the k-th of them at position base + k, and a bound of each sum's fp32
    error.  q [T, hq, d], lse [T, hq], k [l, hkv, d] float64."""
    l, hkv, d = k.shape
    g = q.shape[1] // hkv
    out, err = np.zeros(l), np.zeros(l)
    e = 2.0 ** -24
    for n, t in enumerate(rows):
        seen = base + n + 1
        for h in range(q.shape[1]):
            if lse[t, h] == -np.inf:
                continue
            kk = k[:seen, h // g]
            s = kk @ q[t, h] * scale
            w = np.exp(s - lse[t, h])
            # argument: d products and additions in fp32, then one multiply-add in base 2 of rounded factors; 2^x: 2^-22 of itself
            arg = d * e * (np.abs(kk) @ np.abs(q[t, h])) * scale + 4 * e * (np.abs(s) + abs(lse[t, h]))
            out[:seen] += w
            err[:seen] += w * (arg + 4 * e)
    return out, err + out * e * (len(rows) * q.shape[1])


def evict(w, length, budget, sinks, recent):
    """Positions that stay."""
    if length <= budget:
        return list(range(length))
    free = list(range(sinks, length - recent))
    key = [float("-inf") if np.isnan(w[p]) else float(w[p]) for p in free]
    order = sorted(range(len(free)), key=lambda i: (np.isnan(w[free[i]]), -key[i], free[i]))
    heavy = {free[i] for i in order[:budget - sinks - recent]}
    return [p for p in range(length) if p < sinks or p >= length - recent or p in heavy]
