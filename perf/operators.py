"""What is measured of the serving operators around the path-composed MoE layer: attention over packed prompts,
attention of drafted tokens over a paged cache, the cache's own page operations, and token scores from logits.

``own = False`` computes every operator in its plain form (elementary torch operations in fp32, rounded once at the end);
``own = True`` makes the calls a user makes.  Both take what ``prepare`` gives.  Nothing in ``run`` synchronises."""
from __future__ import annotations

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the fp32 layer's 64 tokens as four short prompts: latency of the smallest call
        dict(name="prompt-tiny-f32", op="prompt", dtype="f32", hq=8, hkv=2, d=64, lens="1,17,45,1"),
        # an ordinary prefill batch of 4096 tokens with 32 heads on 8: ragged prompts, one of them empty, packed
        dict(name="prompt-packed", op="prompt", dtype="bf16", hq=32, hkv=8, d=128, lens="1531,64,0,977,1,1523"),
        # one long prompt with as many kv heads as heads: the largest prefill batch of the configurations
        dict(name="prompt-long", op="prompt", dtype="bf16", hq=16, hkv=16, d=128, lens="16384"),
        # a handful of drafted tokens over short contexts in fp32 (one sequence has no context yet)
        dict(name="tree-small-f32", op="cached", dtype="f32", hq=4, hkv=4, d=64, page=16, ctx="301,0,77", add="7,5,7", tree=True),
        # the decode batch of 32 sequences, one token each, contexts of a chat server
        dict(name="decode-32", op="cached", dtype="bf16", hq=32, hkv=8, d=128, page=64, add=",".join(["1"] * 32), tree=False,
             ctx="4095,1200,733,2048,3001,512,64,2777,1999,3500,150,900,4000,1024,2500,1,3333,600,1750,2222,80,3900,1333,450,2900,1100,3700,260,1600,3100,2400,1900"),
        # trees of up to 48 drafted tokens verified at once over contexts of a few thousand
        dict(name="tree-48", op="cached", dtype="bf16", hq=32, hkv=8, d=128, page=64, tree=True,
             ctx="4050,3011,2500,1777,905,3600,2049,1290", add="48,33,48,17,48,40,48,25"),
        # two users with very long contexts, one token each: the cache read alone
        dict(name="decode-long", op="cached", dtype="bf16", hq=32, hkv=8, d=128, page=16, ctx="131071,100003", add="1,1", tree=False),
        # one turn of drafting: room for the drafts, their rows written, the accepted ones kept, rolled back
        dict(name="cache-turn", op="turn", dtype="bf16", hkv=8, d=128, page=16, layers=8,
             ctx="4050,3011,2500,1777,905,3600,2049,1290", add="48,33,48,17,48,40,48,25", keep="5,1,0,3,9,2,4,1"),
        # best-of-n: eight prompts forked four ways, grown by a token, three of four dropped, the pool compacted
        dict(name="cache-fork", op="fork", dtype="bf16", hkv=8, d=128, page=64, layers=4, ctx="2050,1811,1500,777,905,1600,2049,1290", ways=4),
        # scores of a decode batch: 32 rows, 32000 words
        dict(name="scores-decode", op="scores", dtype="bf16", rows=32, vocab=32000, top=5, banned=0.0),
        # scores of a whole prefill batch (prompt log probabilities)
        dict(name="scores-prompt", op="scores", dtype="bf16", rows=4096, vocab=32000, top=5, banned=0.0),
        # a few rows over a large vocabulary in fp32, most words banned by a grammar, twenty alternatives
        dict(name="scores-wide-f32", op="scores", dtype="f32", rows=7, vocab=151936, top=20, banned=0.7),
    ]


def _loguniform(rng, lo, hi):
    return int(min(hi, max(lo, round(lo * (hi / lo) ** rng.random()))))


def _text(v):
    return ",".join(str(int(x)) for x in v)


def _ints(s):
    return [int(x) for x in str(s).split(",")]


def draw(rng):
    op = rng.choice(["prompt", "prompt", "cached", "cached", "cached", "turn", "fork", "scores", "scores"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    if op == "prompt":
        hq = hkv * rng.choice([1, 2, 3, 4, 7])
        hq = hq if hq <= 32 else hkv * 4
        n = _loguniform(rng, 1, 12)
        most = 2048 if dtype == "f32" else 16384 if hq <= 16 else 8192
        total = _loguniform(rng, 16, most)
        cuts = sorted(rng.randint(0, total) for _ in range(n - 1))
        lens = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        return dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, lens=_text(lens))
    if op == "cached":
        hq = hkv * rng.choice([1, 2, 4, 7, 8])
        hq = hq if hq <= 32 else hkv * 4
        tree = rng.random() < 0.6
        n = _loguniform(rng, 1, 32)
        longest = _loguniform(rng, 1, max(1, min(131072, 160000 // n) // (4 if dtype == "f32" else 1)))
        ctx = [rng.randint(0, longest) for _ in range(n)]
        add = [rng.randint(1, 64) if tree else 1 for _ in range(n)]
        return dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, page=rng.choice([16, 32, 64, 128]), ctx=_text(ctx), add=_text(add), tree=tree)
    if op == "turn":
        n = _loguniform(rng, 1, 24)
        longest = _loguniform(rng, 1, 30000 // n)
        ctx = [rng.randint(1, longest) for _ in range(n)]
        add = [rng.randint(1, 64) for _ in range(n)]
        keep = [rng.randint(0, min(a, 12)) for a in add]
        return dict(op=op, dtype=dtype, hkv=hkv, d=d, page=rng.choice([16, 32, 64]), layers=rng.randint(1, 8), ctx=_text(ctx), add=_text(add), keep=_text(keep))
    if op == "fork":
        n = _loguniform(rng, 1, 16)
        longest = _loguniform(rng, 2, 15000 // n)
        ctx = [rng.randint(1, longest) for _ in range(n)]
        return dict(op=op, dtype=dtype, hkv=hkv, d=d, page=rng.choice([16, 32, 64]), layers=rng.randint(1, 4), ctx=_text(ctx), ways=rng.randint(2, 6))
    rows = _loguniform(rng, 1, 4096)
    vocab = _loguniform(rng, 40, min(160000, 120_000_000 // rows))
    return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, top=rng.choice([0, 1, 5, 8, 20, 32]), banned=rng.choice([0.0, 0.0, 0.5, 0.95]))


# -------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, std=1.0):
    # drawn in the storage type's own fp32 and rounded once
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device=DEV)


def _cu(lens):
    return _i32(np.concatenate([[0], np.cumsum(lens)]))


def _tree_mask(rng, add):
    """Ancestors of every drafted token (itself among them) as bits: word w, bit b of a row = draft 32 w + b of its sequence."""
    words = max(1, (max(add) + 31) // 32)
    rows = []
    for n in add:
        seen = []
        for j in range(n):
            parent = int(rng.integers(-1, j)) if j else -1     # -1: hangs on the context
            bits = (seen[parent] if parent >= 0 else 0) | (1 << j)
            seen.append(bits)
            rows.append([(bits >> (32 * w)) & 0xFFFFFFFF for w in range(words)])
    return torch.tensor(np.asarray(rows, dtype=np.uint32).view(np.int32).reshape(-1, words), device=DEV)


class _Pool:
    """A page pool as a server has it in hand: K and V pages of every layer and the bookkeeping, int32, in one buffer
    (lengths, then reference counts, then page tables)."""

    def __init__(self, g, dtype, layers, pages, page, hkv, d, seqs, slots):
        self.layers, self.pages, self.page, self.hkv, self.d, self.seqs, self.slots = layers, pages, page, hkv, d, seqs, slots
        self.dtype = dtype
        self.k = _randn(g, (layers, pages, hkv, page, d), dtype)
        self.v = _randn(g, (layers, pages, hkv, page, d), dtype)
        self.book = torch.zeros(seqs + pages + seqs * slots, dtype=torch.int32, device=DEV)
        self.len, self.ref, self.table = self.views(self.book)
        self.table.fill_(-1)
        self.handle = None
        if own:
            from paper_2609_01024_b200 import binding as B
            self.handle = B.PagedCache(layers=layers, pages=pages, page_size=page, kv_heads=hkv, head_dim=d, max_seqs=seqs,
                                       max_pages=slots, dtype=_pc(dtype), k=self.k, v=self.v, book=self.book)

    def views(self, book):
        a, b = self.seqs, self.seqs + self.pages
        return book[:a], book[a:b], book[b:].view(self.seqs, self.slots)

    def fill(self, lens, page_ids):
        """Sequences 0.. of the given lengths over the given page ids, in order."""
        ref = np.zeros(self.pages, np.int32)
        table = np.full((self.seqs, self.slots), -1, np.int32)
        at = 0
        for s, n in enumerate(lens):
            m = (n + self.page - 1) // self.page
            table[s, :m] = page_ids[at:at + m]
            at += m
        ref[page_ids[:at]] = 1
        self.len[:len(lens)].copy_(_i32(lens))
        self.ref.copy_(_i32(ref))
        self.table.copy_(_i32(table))
        return at


def _pc(dtype):
    from paper_2609_01024_b200 import binding as B
    return B.PCOMOE_BF16 if dtype == torch.bfloat16 else B.PCOMOE_FP32


def _pages_of(n, page):
    return (n + page - 1) // page


def prepare(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    op = case["op"]
    dt = TYPES[case["dtype"]]
    s = dict(case=case, op=op)
    if op == "prompt":
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        lens = _ints(case["lens"])
        T = sum(lens)
        # q, k and v are column ranges of one fused projection's output, as a model has them
        qkv = _randn(g, (T, (hq + 2 * hkv) * d), dt, 1.25)
        s |= dict(T=T, cu=_cu(lens), q=qkv[:, :hq * d].unflatten(1, (hq, d)), k=qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)),
                  v=qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d)))
        if own:
            from paper_2609_01024_b200 import binding as B
            s["attn"] = B.Attention(q_heads=hq, kv_heads=hkv, head_dim=d, max_tokens=T, max_seqs=len(lens), dtype=_pc(dt))
    elif op == "cached":
        hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
        ctx, add = _ints(case["ctx"]), _ints(case["add"])
        full = [c + a for c, a in zip(ctx, add)]
        need = sum(_pages_of(n, page) for n in full)
        slots = _pages_of(max(full), page)
        pool = _Pool(g, dt, 1, need + 8, page, hkv, d, len(ctx), slots)
        pool.fill(full, rng.permutation(need + 8))
        T = sum(add)
        s |= dict(T=T, pool=pool, cu=_cu(add), seqs=_i32(np.arange(len(ctx))), q=_randn(g, (T, hq, d), dt, 1.25), n_max=max(add), l_max=max(full),
                  mask=_tree_mask(rng, add) if case["tree"] else None)
        if own:
            from paper_2609_01024_b200 import binding as B
            s["attn"] = B.Attention(q_heads=hq, kv_heads=hkv, head_dim=d, max_tokens=T, max_seqs=len(ctx), dtype=_pc(dt))
    elif op == "turn":
        hkv, d, page, layers = case["hkv"], case["d"], case["page"], case["layers"]
        ctx, add, keep = _ints(case["ctx"]), _ints(case["add"]), _ints(case["keep"])
        need = sum(_pages_of(c + a, page) for c, a in zip(ctx, add))
        pool = _Pool(g, dt, layers, need + 8, page, hkv, d, len(ctx), _pages_of(max(c + a for c, a in zip(ctx, add)), page))
        pool.fill(ctx, rng.permutation(need + 8))
        T = sum(add)
        idx = np.full((len(ctx), max(1, max(keep))), -1, np.int32)
        for i, (a, m) in enumerate(zip(add, keep)):
            idx[i, :m] = np.sort(rng.permutation(a)[:m])      # a path of a tree: ascending
        s |= dict(T=T, pool=pool, cu=_cu(add), add=_i32(add), ctx=_i32(ctx), seqs=_i32(np.arange(len(ctx))), n_max=max(add),
                  k=_randn(g, (layers, T, hkv, d), dt), v=_randn(g, (layers, T, hkv, d), dt), keep=_i32(idx), n_keep=_i32(keep))
    elif op == "fork":
        hkv, d, page, layers, ways = case["hkv"], case["d"], case["page"], case["layers"], case["ways"]
        ctx = _ints(case["ctx"])
        n = len(ctx)
        used = sum(_pages_of(c, page) for c in ctx)
        pool = _Pool(g, dt, layers, 2 * used + 2 * n * ways + 2, page, hkv, d, n * (1 + ways), _pages_of(max(ctx) + 1, page))
        pool.fill(ctx, 2 * rng.permutation(used))             # every other page of the low part is taken
        kids = n + np.arange(n * ways)
        s |= dict(pool=pool, parents=_i32(np.repeat(np.arange(n), ways)), kids=_i32(kids), one=_i32(np.ones(n * ways)),
                  losers=_i32(kids.reshape(n, ways)[:, 1:].reshape(-1)), zero=_i32(np.zeros(n * (ways - 1))), saved=pool.book.clone())
    else:
        rows, vocab, top = case["rows"], case["vocab"], min(case["top"], case["vocab"])
        # a few likely words over a broad background
        x = torch.randn((rows, vocab), generator=g, device=DEV) * 2.5
        hot = torch.randint(0, vocab, (rows, 12), generator=g, device=DEV)
        x.scatter_add_(1, hot, 6.0 + 2.0 * torch.randn((rows, 12), generator=g, device=DEV))
        if case["banned"] > 0:
            x.masked_fill_(torch.rand((rows, vocab), generator=g, device=DEV) < case["banned"], float("-inf"))
        tokens = torch.where(torch.rand((rows,), generator=g, device=DEV) < 0.5, hot[:, 0], torch.randint(0, vocab, (rows,), generator=g, device=DEV))
        s |= dict(x=x.to(dt), tokens=tokens.to(torch.int32), top=top)
        if own:
            from paper_2609_01024_b200 import binding as B
            s["scores"] = B.TokenScores(max_tokens=rows, top_n=top)
    return s


# --------------------------------------------------------------------------------------------------- plain forms

def _rows_of(cu, T):
    """Sequence and place inside it of every packed row."""
    t = torch.arange(T, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(cu[1:], t, right=True)
    return seq, t.long() - cu.long()[seq]


def _softmax_rows(scores, v):
    """softmax over the last axis (-inf where nothing may be seen), times v; rows with nothing to see give 0 and -inf."""
    m = scores.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = scores.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o, (m + total.log()).squeeze(-1)


def _plain_prompt(s):
    c = s["case"]
    hq, hkv, d, T = c["hq"], c["hkv"], c["d"], s["T"]
    seq, at = _rows_of(s["cu"], T)
    q = s["q"].float().reshape(T, hkv, hq // hkv, d).permute(1, 2, 0, 3)
    k = s["k"].float().permute(1, 2, 0).unsqueeze(1)
    v = s["v"].float().permute(1, 0, 2).unsqueeze(1)
    scores = torch.matmul(q, k).mul_(d ** -0.5)
    hidden = (seq[:, None] != seq[None, :]) | (at[None, :] > at[:, None])
    o, lse = _softmax_rows(scores.masked_fill_(hidden, float("-inf")), v)
    return o.permute(2, 0, 1, 3).reshape(T, hq, d).to(s["q"].dtype), lse.permute(2, 0, 1).reshape(T, hq)


def _plain_cached(s):
    c, pool = s["case"], s["pool"]
    hq, hkv, d, T, page = c["hq"], c["hkv"], c["d"], s["T"], pool.page
    n = s["seqs"].numel()
    seq, at = _rows_of(s["cu"], T)
    p = torch.arange(s["l_max"], device=DEV)
    pages = pool.table[s["seqs"].long()][:, p // page].clamp(min=0).long()                       # [n, l_max]
    k = pool.k[0][pages, :, p % page].float()                                                    # [n, l_max, hkv, d]
    v = pool.v[0][pages, :, p % page].float()
    length = pool.len[s["seqs"].long()].long()
    base = length - (s["cu"][1:] - s["cu"][:-1]).long()
    q = torch.zeros((n, s["n_max"], hq, d), device=DEV)
    q[seq, at] = s["q"].float()
    q = q.view(n, s["n_max"], hkv, hq // hkv, d).permute(0, 2, 3, 1, 4)
    scores = torch.matmul(q, k.permute(0, 2, 3, 1).unsqueeze(2)).mul_(d ** -0.5)               # [n, hkv, g, n_max, l_max]
    m = p[None, :] - base[:, None]                                                               # draft number of a position
    if s["mask"] is None:
        seen = m[:, None, :] <= torch.arange(s["n_max"], device=DEV)[None, :, None]
    else:
        bits = torch.zeros((n, s["n_max"], s["mask"].shape[1]), dtype=torch.int32, device=DEV)
        bits[seq, at] = s["mask"]
        word = torch.gather(bits, 2, (m.clamp(0, 32 * bits.shape[2] - 1) // 32)[:, None, :].expand(-1, s["n_max"], -1))
        seen = ((word >> (m.clamp(min=0) % 32)[:, None, :]) & 1).bool() | (m < 0)[:, None, :]
    seen = seen & (p[None, :] < length[:, None])[:, None, :]
    o, lse = _softmax_rows(scores.masked_fill_(~seen[:, None, None], float("-inf")), v.permute(0, 2, 1, 3).unsqueeze(2))
    o = o.permute(0, 3, 1, 2, 4).reshape(n, s["n_max"], hq, d)[seq, at]
    return o.to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(n, s["n_max"], hq)[seq, at]


def _excl(x):
    return x.cumsum(0) - x


def _plain_reserve(pool, seqs, add, most):
    """Grows sequences: the lowest free pages in call order, a shared last page copied before the first new row.  `most`: at
    most so many pages are added to one sequence."""
    page = pool.page
    i = seqs.long()
    old = pool.len[i].long()
    new = old + add.long()
    have, want = (old + page - 1) // page, (new + page - 1) // page
    slot = (old // page).clamp(max=pool.slots - 1)
    last = pool.table[i, slot].long().clamp(min=0)
    cut = (old % page > 0) & (add > 0)
    before = ((last[:, None] == last[None, :]) & cut[None, :]).long().tril(-1).sum(1)
    copy = cut & (pool.ref[last].long() - before > 1)
    count = want - have + copy.long()
    first = _excl(count)
    free = (pool.ref == 0).long().cumsum(0)
    j = torch.arange(most + 1, device=DEV)[None, :]
    got = torch.searchsorted(free, (first[:, None] + j + 1).reshape(-1)).view(-1, most + 1).clamp(max=pool.pages - 1)
    mine = j < count[:, None]
    to = (have - copy.long())[:, None] + j
    table = torch.cat([pool.table, pool.table.new_zeros((pool.seqs, most + 2))], 1)
    table[i[:, None], torch.where(mine, to, torch.full_like(to, pool.slots + most + 1))] = got.int()
    pool.table.copy_(table[:, :pool.slots])
    ref = torch.cat([pool.ref, pool.ref.new_zeros(1)])
    ref.index_add_(0, torch.where(mine, got, torch.full_like(got, pool.pages)).reshape(-1), torch.ones_like(got).int().reshape(-1))
    ref.index_add_(0, torch.where(copy, last, torch.full_like(last, pool.pages)), -torch.ones_like(last).int())
    pool.ref.copy_(ref[:-1])
    pool.len[i] = new.int()
    # sequences without a copy repeat the first one that has one (or move a page onto itself where none has)
    f = copy.int().argmax()
    src = torch.where(copy, last, last[f])
    dst = torch.where(copy, got[:, 0], torch.where(copy[f], got[f, 0], last[f]))
    pool.k[:, dst] = pool.k[:, src]
    pool.v[:, dst] = pool.v[:, src]


def _plain_trim(pool, seqs, lens):
    i = seqs.long()
    keep = (lens.long() + pool.page - 1) // pool.page
    row = pool.table[i]
    gone = (torch.arange(pool.slots, device=DEV)[None, :] >= keep[:, None]) & (row >= 0)
    ref = torch.cat([pool.ref, pool.ref.new_zeros(1)])
    ref.index_add_(0, torch.where(gone, row.long(), torch.full_like(row.long(), pool.pages)).reshape(-1), -torch.ones_like(row).reshape(-1))
    pool.ref.copy_(ref[:-1])
    pool.table[i] = torch.where(gone, torch.full_like(row, -1), row)
    pool.len[i] = lens


def _plain_turn(s):
    pool, T = s["pool"], s["T"]
    i = s["seqs"].long()
    _plain_reserve(pool, s["seqs"], s["add"], s["n_max"] // pool.page + 2)
    seq, at = _rows_of(s["cu"], T)
    base = pool.len[i].long() - s["add"].long()
    p = base[seq] + at
    where = pool.table[i[seq], p // pool.page].long()
    pool.k[:, where, :, p % pool.page] = s["k"].permute(1, 0, 2, 3)
    pool.v[:, where, :, p % pool.page] = s["v"].permute(1, 0, 2, 3)
    # the accepted rows move up behind the context
    m = torch.arange(s["keep"].shape[1], device=DEV)[None, :].expand_as(s["keep"])
    used = m < s["n_keep"][:, None]
    src = base[:, None] + torch.where(used, s["keep"].long(), torch.zeros_like(m))
    dst = base[:, None] + torch.where(used, m, torch.zeros_like(m))
    from_page, to_page = (pool.table[i[:, None], x // pool.page].long() for x in (src, dst))
    k_rows, v_rows = (x[:, from_page, :, src % pool.page] for x in (pool.k, pool.v))
    same_k, same_v = (x[:, to_page[:, :1], :, (dst % pool.page)[:, :1]] for x in (pool.k, pool.v))
    first_used = used[:, :1, None, None, None]
    head_k, head_v = torch.where(first_used, k_rows[:, :1], same_k), torch.where(first_used, v_rows[:, :1], same_v)
    # unused places repeat the first one: every write to a place carries the same value
    at_page = torch.where(used, to_page, to_page[:, :1])
    at_row = torch.where(used, dst, dst[:, :1]) % pool.page
    pool.k[:, at_page, :, at_row] = torch.where(used[:, :, None, None, None], k_rows, head_k)
    pool.v[:, at_page, :, at_row] = torch.where(used[:, :, None, None, None], v_rows, head_v)
    _plain_trim(pool, s["seqs"], (base + s["n_keep"].long()).int())
    kept = pool.book.clone()
    _plain_trim(pool, s["seqs"], s["ctx"])
    return dict(k=pool.k, v=pool.v, kept=kept, book=pool.book)


def _plain_fork(s):
    pool = s["pool"]
    row = pool.table[s["parents"].long()]
    pool.table[s["kids"].long()] = row
    pool.len[s["kids"].long()] = pool.len[s["parents"].long()]
    ref = torch.cat([pool.ref, pool.ref.new_zeros(1)])
    ref.index_add_(0, torch.where(row >= 0, row, torch.full_like(row, pool.pages)).long().reshape(-1), torch.ones_like(row).reshape(-1))
    pool.ref.copy_(ref[:-1])
    _plain_reserve(pool, s["kids"], s["one"], 2)
    grown = pool.book.clone()
    _plain_trim(pool, s["losers"], s["zero"])
    # compaction: the live pages from `used` on go, in order, to the free places below it
    live = pool.ref > 0
    used = live.sum()
    ids = torch.arange(pool.pages, device=DEV)
    high = live & (ids >= used)
    holes = (~live & (ids < used)).long().cumsum(0)
    to = torch.where(high, torch.searchsorted(holes, high.long().cumsum(0)), ids)
    comes = torch.cat([ids, ids[:1]])
    comes[torch.where(high, to, torch.full_like(ids, pool.pages))] = ids
    comes = comes[:-1]
    pool.k.copy_(pool.k[:, comes])
    pool.v.copy_(pool.v[:, comes])
    ref = pool.ref[comes] * (ids < used)
    pool.ref.copy_(ref)
    pool.table.copy_(torch.where(pool.table >= 0, to[pool.table.long().clamp(min=0)].int(), pool.table))
    packed = pool.book.clone()
    pool.book.copy_(s["saved"])
    return dict(k=pool.k, v=pool.v, grown=grown, packed=packed)


def _plain_scores(s):
    x = s["x"].float()
    m = x.amax(1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    z = (x - m).exp().sum(1, keepdim=True).log() + m
    z = torch.where(torch.isinf(z), torch.zeros_like(z), z)      # a row without an eligible word
    lp = x - z
    entropy = -(lp.exp() * torch.where(torch.isinf(lp), torch.zeros_like(lp), lp)).sum(1)
    given = lp.gather(1, s["tokens"].long()[:, None])[:, 0]
    if not s["top"]:
        return dict(logprob=given, entropy=entropy)
    best, ids = torch.sort(x, dim=1, descending=True, stable=True)
    best, ids = best[:, :s["top"]], ids[:, :s["top"]].int()
    return dict(logprob=given, entropy=entropy, top=best - z, ids=torch.where(torch.isinf(best), torch.full_like(ids, -1), ids))


# ----------------------------------------------------------------------------------------------- the user's calls

def _own_turn(s):
    c = s["pool"].handle
    c.reserve(s["seqs"], s["add"])
    c.write(s["k"], s["v"], s["seqs"], s["cu"])
    c.keep(s["seqs"], s["cu"], s["keep"], s["n_keep"])
    kept = s["pool"].book.clone()
    c.trim(s["seqs"], s["ctx"])
    return dict(k=c.k, v=c.v, kept=kept, book=s["pool"].book)


def _own_fork(s):
    c, pool = s["pool"].handle, s["pool"]
    c.fork(s["parents"], s["kids"])
    c.reserve(s["kids"], s["one"])
    grown = pool.book.clone()
    c.trim(s["losers"], s["zero"])
    c.compact()
    packed = pool.book.clone()
    pool.book.copy_(s["saved"])
    return dict(k=c.k, v=c.v, grown=grown, packed=packed)


def _own_scores(s):
    logprob, entropy, ids, top = s["scores"].score(s["x"], s["tokens"])
    return dict(logprob=logprob, entropy=entropy, top=top, ids=ids) if s["top"] else dict(logprob=logprob, entropy=entropy)


def run(s):
    op = s["op"]
    if own:
        if op == "prompt":
            return s["attn"].prompt(s["q"], s["k"], s["v"], s["cu"])
        if op == "cached":
            return s["attn"].cached(s["q"], s["pool"].handle, 0, s["seqs"], s["cu"], s["mask"])
        return {"turn": _own_turn, "fork": _own_fork, "scores": _own_scores}[op](s)
    return {"prompt": _plain_prompt, "cached": _plain_cached, "turn": _plain_turn, "fork": _plain_fork, "scores": _plain_scores}[op](s)


# ------------------------------------------------------------------------------------------------------- the work

def work(case):
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "prompt":
        lens = _ints(case["lens"])
        T, hq, hkv, d = sum(lens), case["hq"], case["hkv"], case["d"]
        return dict(bytes=e * T * d * (2 * hq + 2 * hkv) + 4 * T * hq, flops=4 * d * hq * sum(n * (n + 1) // 2 for n in lens))
    if op == "cached":
        ctx, add = _ints(case["ctx"]), _ints(case["add"])
        hq, hkv, d, T = case["hq"], case["hkv"], case["d"], sum(add)
        seen = sum(a * c + a * (a + 1) // 2 for c, a in zip(ctx, add))       # of a chain; a tree sees no more
        rows = sum(ctx) + T
        return dict(bytes=2 * e * hkv * d * rows + 2 * e * T * hq * d + 4 * T * hq + 4 * rows // case["page"], flops=4 * d * hq * seen)
    if op == "turn":
        row = 2 * e * case["hkv"] * case["d"] * case["layers"]               # K and V of a token in all layers
        return dict(bytes=2 * row * (sum(_ints(case["add"])) + sum(_ints(case["keep"]))), flops=0)
    if op == "fork":
        page, ways = case["page"], case["ways"]
        ctx = _ints(case["ctx"])
        per = 2 * e * case["hkv"] * case["d"] * case["layers"] * page
        live = {2 * i for i in range(sum(_pages_of(c, page) for c in ctx))}
        at = 1
        copies = 0
        for c in ctx:
            for w in range(ways):
                copies += 1 if c % page else 0
                if w == 0:
                    live.add(at)                                              # the winner's own page (copied or new)
                at += 2
        moves = sum(1 for p in live if p >= len(live))
        return dict(bytes=2 * per * (copies + moves), flops=0)
    rows, vocab, top = case["rows"], case["vocab"], min(case["top"], case["vocab"])
    return dict(bytes=e * rows * vocab + 4 * rows * (3 + 2 * top), flops=4 * rows * vocab)


# ------------------------------------------------------------------------------------------ the definition, 64 bits

def _attend64(q, k, v, seen, scale):
    """q [n,d], k and v [l,d], seen [n,l] (None: everything), in fp64."""
    x = (q @ k.T) * scale
    if seen is not None:
        x = torch.where(seen, x, x.new_tensor(float("-inf")))
    lse = torch.logsumexp(x, -1)
    w = torch.where(torch.isinf(lse)[:, None], torch.zeros_like(x), (x - lse[:, None]).exp())
    return w @ v, lse


def _exact_prompt(s):
    c = s["case"]
    g = c["hq"] // c["hkv"]
    o = torch.zeros((s["T"], c["hq"], c["d"]), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["T"], c["hq"]), dtype=torch.float64, device=DEV)
    a = 0
    for n in _ints(c["lens"]):
        for h in range(c["hq"]):
            for lo in range(0, n, 2048):
                hi = min(n, lo + 2048)
                seen = torch.arange(hi, device=DEV)[None, :] <= torch.arange(lo, hi, device=DEV)[:, None]
                o[a + lo:a + hi, h], lse[a + lo:a + hi, h] = _attend64(s["q"][a + lo:a + hi, h].double(), s["k"][a:a + hi, h // g].double(),
                                                                     s["v"][a:a + hi, h // g].double(), seen, c["d"] ** -0.5)
        a += n
    return o, lse


def _exact_cached(s):
    c, pool = s["case"], s["pool"]
    g, T = c["hq"] // c["hkv"], s["T"]
    o = torch.zeros((T, c["hq"], c["d"]), dtype=torch.float64, device=DEV)
    lse = torch.zeros((T, c["hq"]), dtype=torch.float64, device=DEV)
    table = pool.table.cpu().numpy()
    words = None if s["mask"] is None else s["mask"].cpu().numpy().view(np.uint32)
    a = 0
    for i, (past, n) in enumerate(zip(_ints(c["ctx"]), _ints(c["add"]))):
        pages = torch.tensor(table[i, :_pages_of(past + n, pool.page)].astype(np.int64), device=DEV)
        k, v = (x[0, pages].transpose(1, 2).reshape(-1, c["hkv"], c["d"])[:past + n] for x in (pool.k, pool.v))
        see = np.zeros((n, past + n), bool)
        see[:, :past] = True
        for j in range(n):
            for m in range(n):
                see[j, past + m] = m <= j if words is None else bool((int(words[a + j, m // 32]) >> (m % 32)) & 1)
        see = torch.tensor(see, device=DEV)
        for h in range(c["hq"]):
            o[a:a + n, h], lse[a:a + n, h] = _attend64(s["q"][a:a + n, h].double(), k[:, h // g].double(), v[:, h // g].double(), see, c["d"] ** -0.5)
        a += n
    return o, lse


class _Book:
    """The bookkeeping on the host, one page at a time."""

    def __init__(self, pool):
        self.pool = pool
        n, r, t = (x.cpu().numpy().copy() for x in (pool.len, pool.ref, pool.table))
        self.len, self.ref, self.table = n, r, t

    def take(self):
        p = int(np.flatnonzero(self.ref == 0)[0])
        self.ref[p] = 1
        return p

    def reserve(self, seqs, add):
        page, copies = self.pool.page, []
        for s, n in zip(seqs, add):
            for at in range(int(self.len[s]), int(self.len[s]) + n):
                slot = at // page
                p = self.table[s, slot]
                if at % page == 0:
                    self.table[s, slot] = self.take()
                elif self.ref[p] > 1:
                    new = self.take()
                    self.ref[p] -= 1
                    copies.append((int(p), new))
                    self.table[s, slot] = new
            self.len[s] += n
        return copies

    def trim(self, seqs, lens):
        for s, n in zip(seqs, lens):
            for slot in range(_pages_of(n, self.pool.page), self.pool.slots):
                if self.table[s, slot] >= 0:
                    self.ref[self.table[s, slot]] -= 1
                    self.table[s, slot] = -1
            self.len[s] = n

    def flat(self):
        return torch.tensor(np.concatenate([self.len, self.ref, self.table.reshape(-1)]), device=DEV)


def _exact_turn(s):
    c, pool = s["case"], s["pool"]
    ctx, add, keep = (_ints(c[x]) for x in ("ctx", "add", "keep"))
    b = _Book(pool)
    b.reserve(range(len(ctx)), add)
    out = [pool.k.clone(), pool.v.clone()]
    new = [s["k"], s["v"]]
    idx = s["keep"].cpu().numpy()
    a = 0
    for i, (past, n) in enumerate(zip(ctx, add)):
        place = [(int(b.table[i, p // pool.page]), p % pool.page) for p in range(past, past + n)]
        for x, y in zip(out, new):
            for j, (p, r) in enumerate(place):
                x[:, p, :, r] = y[:, a + j]
            for j in range(keep[i]):
                (p, r) = place[j]
                x[:, p, :, r] = y[:, a + int(idx[i, j])]
        a += n
    b.trim(range(len(ctx)), [x + y for x, y in zip(ctx, keep)])
    kept = b.flat()
    b.trim(range(len(ctx)), ctx)
    return dict(k=out[0].double(), v=out[1].double(), kept=kept, book=b.flat())


def _exact_fork(s):
    pool = s["pool"]
    b = _Book(pool)
    for p, kid in zip(s["parents"].tolist(), s["kids"].tolist()):
        b.table[kid], b.len[kid] = b.table[p], b.len[p]
        b.ref[b.table[p][b.table[p] >= 0]] += 1
    moves = b.reserve(s["kids"].tolist(), s["one"].tolist())
    grown = b.flat()
    b.trim(s["losers"].tolist(), [0] * s["losers"].numel())
    live = [int(p) for p in np.flatnonzero(b.ref > 0)]
    holes = [p for p in range(len(live)) if b.ref[p] == 0]
    for old, new in zip([p for p in live if p >= len(live)], holes):
        moves.append((old, new))
        b.ref[new], b.ref[old] = b.ref[old], 0
        b.table[b.table == old] = new
    out = [pool.k.clone(), pool.v.clone()]
    for x in out:
        for old, new in moves:
            x[:, new] = x[:, old]
    return dict(k=out[0].double(), v=out[1].double(), grown=grown, packed=b.flat())


def _exact_scores(s):
    x = s["x"].double()
    z = torch.logsumexp(x, 1)
    z = torch.where(torch.isinf(z), torch.zeros_like(z), z)
    lp = x - z[:, None]
    entropy = torch.special.entr(lp.exp()).sum(1)
    out = dict(logprob=lp[torch.arange(len(x), device=DEV), s["tokens"].long()], entropy=entropy)
    if s["top"]:
        # by value, then by the smaller id: every id's number of better ones
        v, ids = torch.sort(x, dim=1, descending=True, stable=True)
        v, ids = v[:, :s["top"]], ids[:, :s["top"]].int()
        out |= dict(top=v - z[:, None], ids=torch.where(torch.isinf(v), torch.full_like(ids, -1), ids))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"prompt": _exact_prompt, "cached": _exact_cached, "turn": _exact_turn, "fork": _exact_fork, "scores": _exact_scores}[case["op"]](s)
