"""Plain 64-bit implementations of the serving operators (attention, paged cache, token scores) for the tests.

Everything is written from the definitions with loops over sequences, heads, pages and rows; nothing is shared with the
library.  Attention and scores return fp64; the cache is a host model whose data are dictionaries of rows."""
import numpy as np
import torch


def attend(q, k, v, seen, scale):
    """One head: q [n,D], k, v [l,D] (fp64), seen [n,l] bool.  Returns o, lse and the weighted mean of |v| (the size that
    rounding errors of the weights scale with).  Values that a row does not see are not touched."""
    n, d = q.shape
    o = torch.zeros(n, d, dtype=torch.float64)
    size = torch.zeros(n, d, dtype=torch.float64)
    lse = torch.full((n,), float("-inf"), dtype=torch.float64)
    for i in range(n):
        at = torch.nonzero(seen[i]).flatten()
        if at.numel() == 0:
            continue
        x = (k[at] @ q[i]) * scale
        lse[i] = torch.logsumexp(x, 0)
        w = torch.exp(x - lse[i])
        o[i] = w @ v[at]
        size[i] = w @ v[at].abs()
    return o, lse, size


def prompt(q, k, v, lens, scale):
    """q [T,Hq,D], k, v [T,Hkv,D] CPU tensors of any type."""
    q, k, v = q.double(), k.double(), v.double()
    T, hq, d = q.shape
    g = hq // k.shape[1]
    o, lse, size = torch.zeros(T, hq, d, dtype=torch.float64), torch.zeros(T, hq, dtype=torch.float64), torch.zeros(T, hq, d, dtype=torch.float64)
    a = 0
    for n in lens:
        seen = torch.tril(torch.ones(n, n, dtype=torch.bool))
        for h in range(hq):
            o[a:a + n, h], lse[a:a + n, h], size[a:a + n, h] = attend(q[a:a + n, h], k[a:a + n, h // g], v[a:a + n, h // g], seen, scale)
        a += n
    return o, lse, size


def cached(q, keys, values, counts, seen, scale):
    """keys, values: per query group [l,Hkv,D]; seen: per group [n,l] bool."""
    q = q.double()
    T, hq, d = q.shape
    o, lse, size = torch.zeros(T, hq, d, dtype=torch.float64), torch.zeros(T, hq, dtype=torch.float64), torch.zeros(T, hq, d, dtype=torch.float64)
    a = 0
    for n, kk, vv, see in zip(counts, keys, values, seen):
        g = hq // kk.shape[1]
        for h in range(hq):
            o[a:a + n, h], lse[a:a + n, h], size[a:a + n, h] = attend(q[a:a + n, h], kk[:, h // g].double(), vv[:, h // g].double(), see, scale)
        a += n
    return o, lse, size


def tree_bits(rng, n):
    """Ancestor rows of a random tree of n drafted tokens: [n,n] bool, itself included."""
    see = np.zeros((n, n), bool)
    for j in range(n):
        parent = int(rng.integers(-1, j)) if j else -1
        if parent >= 0:
            see[j] = see[parent]
        see[j, j] = True
    return see


def pack_bits(rows, words):
    """List of [n,n] bool -> [sum n, words] int32 mask words."""
    out = []
    for see in rows:
        for r in see:
            bits = sum(1 << int(m) for m in np.flatnonzero(r))
            out.append([(bits >> (32 * w)) & 0xFFFFFFFF for w in range(words)])
    return torch.from_numpy(np.asarray(out, dtype=np.uint32).reshape(-1, words).view(np.int32).copy())


class Book:
    """The cache's bookkeeping, one page at a time, in the order that the calls promise."""

    def __init__(self, pages, page, max_seqs, max_pages):
        self.page, self.max_pages = page, max_pages
        self.len = np.zeros(max_seqs, np.int32)
        self.ref = np.zeros(pages, np.int32)
        self.table = np.full((max_seqs, max_pages), -1, np.int32)
        self.moves = []                       # (from, to) of the last call, whole pages

    def need(self, n):
        return -(-n // self.page)

    def take(self):
        p = int(np.flatnonzero(self.ref == 0)[0])
        self.ref[p] = 1
        return p

    def reserve(self, seqs, add):
        self.moves = []
        for s, n in zip(seqs, add):
            for p in range(int(self.len[s]), int(self.len[s]) + n):
                slot, old = p // self.page, self.table[s, p // self.page]
                if p % self.page == 0:
                    self.table[s, slot] = self.take()
                elif self.ref[old] > 1:
                    new = self.take()
                    self.ref[old] -= 1
                    self.moves.append((int(old), new))
                    self.table[s, slot] = new
            self.len[s] += n

    def fork(self, parents, children):
        for p, c in zip(parents, children):
            self.table[c], self.len[c] = self.table[p], self.len[p]
            self.ref[self.table[p][self.table[p] >= 0]] += 1

    def trim(self, seqs, lens):
        for s, n in zip(seqs, lens):
            for slot in range(self.need(n), self.max_pages):
                if self.table[s, slot] >= 0:
                    self.ref[self.table[s, slot]] -= 1
                    self.table[s, slot] = -1
            self.len[s] = n

    def compact(self):
        live = np.flatnonzero(self.ref > 0)
        holes = [p for p in range(len(live)) if self.ref[p] == 0]
        self.moves = list(zip([int(p) for p in live if p >= len(live)], holes))
        for old, new in self.moves:
            self.ref[new], self.ref[old] = self.ref[old], 0
            self.table[self.table == old] = new

    def place(self, s, p):
        return int(self.table[s, p // self.page]), p % self.page


def scores(x, tokens, top):
    """x [T,V] CPU.  Returns logprob, entropy (fp64) and top ids, top log probabilities, by the definition."""
    x = x.double().clone()
    x[~torch.isfinite(x)] = float("-inf")
    T, V = x.shape
    lp, ent = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    ids, best = torch.full((T, top), -1, dtype=torch.int32), torch.full((T, top), float("-inf"), dtype=torch.float64)
    for t in range(T):
        y = x[t] - x[t].max() if torch.isfinite(x[t].max()) else x[t]          # shifted: rows of 1e38 keep their log sum
        z = torch.logsumexp(y, 0)
        if torch.isinf(z):
            z = torch.zeros((), dtype=torch.float64)
        p = torch.exp(y - z)
        ent[t] = -(p[p > 0] * (y - z)[p > 0]).sum()
        tok = int(tokens[t])
        lp[t] = float("nan") if tok >= V else 0.0 if tok < 0 else y[tok] - z
        order = sorted(range(V), key=lambda i: (-float(x[t, i]), i))[:top] if V <= 4096 else \
            np.lexsort((np.arange(V), -x[t].numpy()))[:top].tolist()
        for r, i in enumerate(order):
            if x[t, i] > float("-inf"):
                ids[t, r], best[t, r] = i, y[i] - z
    return lp, ent, ids, best
