"""What is measured of a sampled, drafted decoding turn over a bounded cache: norms and rotation of queries and keys on their
way into the cache, verification of drafted tokens from given random numbers, attention weight accumulated per cached
position, and eviction by it.

``own = False`` computes every operator in its plain form (elementary torch operations); ``own = True`` makes the calls a user
makes.  Both take what ``prepare`` gives.  Nothing in ``run`` synchronises."""
from __future__ import annotations

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------- cases

def listed():
    chat = "4095,1200,733,2048,3001,512,64,2777,1999,3500,150,900,4000,1024,2500,1,3333,600,1750,2222,80,3900,1333,450,2900,1100,3700,260,1600,3100,2400,1900"
    return [
        # four rows of the fp32 type, packed in and out: the smallest call, latency alone
        dict(name="rotate-tiny-f32", op="rotate", dtype="f32", hq=8, hkv=2, d=64, rot=64, pairs="halves", norm=True, into="packed", page=16, ctx="0,0", add="3,1"),
        # a decode step of 32 sequences: keys and values go straight to their pages, far positions
        dict(name="rotate-decode-32", op="rotate", dtype="bf16", hq=32, hkv=8, d=128, rot=128, pairs="halves", norm=True, into="cache", page=64,
             ctx=",".join(str((37 * i) % 300) for i in range(32)), add=",".join(["1"] * 32)),
        # a prefill batch of 16384 tokens, as many kv heads as heads: rotated keys are needed packed and in the cache
        dict(name="rotate-prompt", op="rotate", dtype="bf16", hq=16, hkv=16, d=128, rot=128, pairs="halves", norm=True, into="both", page=64,
             ctx="0,0,0,0,0", add="9001,0,1531,1,5851"),
        # a drafting turn with its chains: 8 drafts and the token before them, in 32 sequences, Mixtral's vocabulary
        dict(name="verify-chain", op="verify", dtype="bf16", vocab=32000, drafts=True, tree=False, add=",".join(["9"] * 32), temp="1.0"),
        # trees of given (not drawn) drafts, some sequences greedy
        dict(name="verify-tree", op="verify", dtype="bf16", vocab=32000, drafts=False, tree=True, add="48,33,48,17,48,40,48,25", temp="0.7,0"),
        # one plain sampling step of a few sequences over a large vocabulary in fp32
        dict(name="verify-wide-f32", op="verify", dtype="f32", vocab=151936, drafts=True, tree=False, add="1,1,5,1,3", temp="0.8"),
        # a few fp32 rows over short contexts
        dict(name="weigh-tiny-f32", op="weigh", dtype="f32", hq=4, hkv=4, d=64, page=16, ctx="301,0,77", add="7,5,7", keep="2,1,3"),
        # the decode batch of 32 sequences, contexts of a chat server
        dict(name="weigh-decode-32", op="weigh", dtype="bf16", hq=32, hkv=8, d=128, page=64, ctx=chat, add=",".join(["1"] * 32), keep=""),
        # two users with very long contexts, the accepted ones of eight drafts each
        dict(name="weigh-long", op="weigh", dtype="bf16", hq=32, hkv=8, d=128, page=16, ctx="131071,100003", add="8,8", keep="4,1"),
        # a whole prompt of 8192 tokens weighed at once after its prefill
        dict(name="weigh-prompt", op="weigh", dtype="bf16", hq=32, hkv=8, d=128, page=64, ctx="0", add="8192", keep=""),
        # a prefill batch written and cut down to a budget each
        dict(name="evict-batch", op="evict", dtype="bf16", hkv=8, d=128, page=64, layers=4, lens="4050,3011,2500,1777,905,3600,2049,1290",
             budget="1024,1024,1024,1024,1024,2048,2000,512", sinks=4, recent=64),
        # one very long prompt cut to a quarter
        dict(name="evict-long", op="evict", dtype="bf16", hkv=8, d=128, page=16, layers=2, lens="131071", budget="32768", sinks=4, recent=256),
    ]


def _loguniform(rng, lo, hi):
    return int(min(hi, max(lo, round(lo * (hi / lo) ** rng.random()))))


def _text(v):
    return ",".join(str(int(x)) for x in v)


def _ints(s):
    return [int(x) for x in str(s).split(",")] if str(s) else []


def draw(rng):
    op = rng.choice(["rotate", "rotate", "verify", "verify", "weigh", "weigh", "weigh", "evict"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 7])
    hq = hq if hq <= 32 else hkv * 4
    if op == "rotate":
        n = _loguniform(rng, 1, 64)
        total = _loguniform(rng, n, 16384 if dtype == "bf16" and hq <= 16 else 8192)
        cuts = sorted(rng.randint(0, total) for _ in range(n - 1))
        add = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        rot = rng.choice([d, d, d // 2, 16, 48])
        return dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, rot=rot, pairs=rng.choice(["halves", "neighbours"]), norm=rng.random() < 0.7,
                    into=rng.choice(["packed", "cache", "both"]), page=rng.choice([16, 32, 64, 128]), ctx=_text(rng.randint(0, 200) for _ in range(n)), add=_text(add))
    if op == "verify":
        tree = rng.random() < 0.4
        n = _loguniform(rng, 1, 48)
        most = 32 if tree else 9
        add = [rng.randint(1, most) for _ in range(n)]
        vocab = _loguniform(rng, 50, min(160000, 9_000_000 // sum(add)))
        temp = rng.choice(["1.0", "0.6", "1.3", "0.9,0", "0"])
        return dict(op=op, dtype=dtype, vocab=vocab, drafts=rng.random() < 0.6, tree=tree, add=_text(add), temp=temp)
    if op == "weigh":
        n = _loguniform(rng, 1, 32)
        long_rows = rng.random() < 0.3
        longest = _loguniform(rng, 1, max(1, (5000 if long_rows else min(131072, 160000 // n)) // (4 if dtype == "f32" else 1)))
        ctx = [rng.randint(0, longest) for _ in range(n)]
        if long_rows:                                           # chunks of a prompt
            most = max(1, 4096 // n // (4 if dtype == "f32" else 1))
            add = [rng.randint(1, most) for _ in range(n)]
            return dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, page=rng.choice([16, 32, 64, 128]), ctx=_text(ctx), add=_text(add), keep="")
        add = [rng.randint(1, 16) for _ in range(n)]
        keep = _text(rng.randint(0, min(a, 6)) for a in add) if rng.random() < 0.6 else ""
        return dict(op=op, dtype=dtype, hq=hq, hkv=hkv, d=d, page=rng.choice([16, 32, 64, 128]), ctx=_text(ctx), add=_text(add), keep=keep)
    n = _loguniform(rng, 1, 16)
    longest = _loguniform(rng, 2, 30000 // n)
    lens = [rng.randint(1, longest) for _ in range(n)]
    sinks, recent = rng.randint(0, 8), rng.choice([0, 1, 16, 64])
    budget = [max(sinks + recent, rng.randint(0, max(1, x))) for x in lens]
    return dict(op=op, dtype=dtype, hkv=hkv, d=d, page=rng.choice([16, 32, 64, 128]), layers=rng.randint(1, 4), lens=_text(lens), budget=_text(budget), sinks=sinks, recent=recent)


# -------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, std=1.0):
    # drawn in fp32 and rounded once to the storage type
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _rand(g, shape):
    return torch.rand(shape, generator=g, device=DEV)


def _i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device=DEV)


def _cu(lens):
    return _i32(np.concatenate([[0], np.cumsum(lens)]))


def _pages_of(n, page):
    return (n + page - 1) // page


def _pc(dtype):
    from paper_2609_01024_b200 import binding as B
    return B.PCOMOE_BF16 if dtype == torch.bfloat16 else B.PCOMOE_FP32


class _Pool:
    """A page pool as a server has it in hand: K and V pages of every layer and the bookkeeping (lengths, reference counts, page
    tables) in one int32 buffer.  The pages of the sequences lie in random order."""

    def __init__(self, g, rng, dtype, layers, page, hkv, d, lens, room, values=True):
        n = len(lens)
        need = sum(_pages_of(x, page) for x in room)
        self.layers, self.pages, self.page, self.hkv, self.d, self.seqs = layers, need + 3, page, hkv, d, n
        self.slots = max(1, max(_pages_of(x, page) for x in room))
        shape = (layers, self.pages, hkv, page, d)
        self.k = _randn(g, shape, dtype) if values else torch.zeros(shape, dtype=dtype, device=DEV)
        self.v = _randn(g, shape, dtype) if values else torch.zeros(shape, dtype=dtype, device=DEV)
        ids = rng.permutation(self.pages)
        ref = np.zeros(self.pages, np.int32)
        table = np.full((n, self.slots), -1, np.int32)
        at = 0
        for s, x in enumerate(lens):
            m = _pages_of(x, page)
            table[s, :m] = ids[at:at + m]
            ref[ids[at:at + m]] = 1
            at += m
        self.book = _i32(np.concatenate([np.asarray(lens), ref, table.reshape(-1)]))
        a, b = n, n + self.pages
        self.len, self.ref, self.table = self.book[:a], self.book[a:b], self.book[b:].view(n, self.slots)
        self.handle = None
        if own:
            from paper_2609_01024_b200 import binding as B
            self.handle = B.PagedCache(layers=layers, pages=self.pages, page_size=page, kv_heads=hkv, head_dim=d, max_seqs=n, max_pages=self.slots,
                                       dtype=_pc(dtype), k=self.k, v=self.v, book=self.book)


def _tree_parents(rng, n):
    """Parents of n drafted rows, the first one given; most hang on a recent one."""
    return [-1] + [int(max(0, j - 1 - rng.geometric(0.5) + 1)) if rng.random() < 0.7 else int(rng.integers(0, j)) for j in range(1, n)]


def _prepare_rotate(case, g, rng, dt):
    hq, hkv, d, rot = case["hq"], case["hkv"], case["d"], case["rot"]
    ctx, add = _ints(case["ctx"]), _ints(case["add"])
    T = sum(add)
    # q, k and v are column ranges of one fused projection's output, as a model has them
    qkv = _randn(g, (T, (hq + 2 * hkv) * d), dt, 1.5)
    start = [0 if c == 0 else int(rng.integers(c, 131072 - a)) for c, a in zip(ctx, add)]       # a place in the cache is no position once rows were evicted
    s = dict(T=T, q=qkv[:, :hq * d].unflatten(1, (hq, d)), k=qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)), v=qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d)),
             position=_i32(np.concatenate([np.arange(a) + x for x, a in zip(start, add)])), cu=_cu(add), eps=1e-6,
             inv_freq=torch.tensor(1e6 ** (-np.arange(rot // 2) / (rot / 2)), dtype=torch.float64, device=DEV),
             q_weight=_randn(g, (d,), dt, 0.2) + 1 if case["norm"] else None, k_weight=_randn(g, (d,), dt, 0.2) + 1 if case["norm"] else None,
             q_out=torch.empty((T, hq, d), dtype=dt, device=DEV), k_out=torch.empty((T, hkv, d), dtype=dt, device=DEV) if case["into"] != "cache" else None)
    if case["into"] != "packed":
        full = [c + a for c, a in zip(ctx, add)]
        s["pool"] = _Pool(g, rng, dt, 1, case["page"], hkv, d, full, full)
        s["seqs"] = _i32(np.arange(len(ctx)))
    if own:
        from paper_2609_01024_b200 import binding as B
        s["rotation"] = B.HeadRotation(q_heads=hq, kv_heads=hkv, head_dim=d, rot_dim=rot, inv_freq=s["inv_freq"], neighbours=case["pairs"] == "neighbours",
                                       q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"], dtype=_pc(dt))
    return s


def _prepare_verify(case, g, rng, dt):
    V, add = case["vocab"], _ints(case["add"])
    T, n = sum(add), len(add)
    first = np.concatenate([[0], np.cumsum(add)])[:-1]
    local = [_tree_parents(rng, a) if case["tree"] else list(range(-1, a - 1)) for a in add]
    up = np.concatenate([np.maximum(0, np.asarray(p)) + f for p, f in zip(local, first)])       # packed row of the parent
    # the target's logits: a few likely words over a broad background, some words banned; the drafter's are near them
    x = torch.randn((T, V), generator=g, device=DEV) * 2.0
    hot = torch.randint(0, V, (T, 12), generator=g, device=DEV)
    x.scatter_add_(1, hot, 6.0 + 2.0 * torch.randn((T, 12), generator=g, device=DEV))
    near = torch.softmax(x + torch.randn((T, V), generator=g, device=DEV) * 0.7, 1)
    x.masked_fill_(_rand(g, (T, V)) < 0.02, float("-inf"))
    up_dev = torch.tensor(up, device=DEV)
    if case["drafts"]:
        tokens = torch.multinomial(near[up_dev], 1, generator=g)[:, 0]          # drawn from the drafter's row of their parent
    else:
        # the best words of the drafter, one after another among siblings
        rank = torch.tensor([sum(1 for m in range(1, j) if p[m] == p[j]) if j else 0 for p in local for j in range(len(p))], device=DEV)
        best = torch.topk(near, min(V, int(rank.max()) + 1), dim=1).indices
        tokens = best[up_dev].gather(1, rank.clamp(max=best.shape[1] - 1)[:, None])[:, 0]
    temps = [float(t) for t in str(case["temp"]).split(",")]
    s = dict(T=T, n=n, cu=_cu(add), tokens=tokens.to(torch.int32), parent=_i32(np.concatenate(local)) if case["tree"] else None, x=x.to(dt),
             near=near if case["drafts"] else None, temperature=torch.tensor([temps[i % len(temps)] for i in range(n)], dtype=torch.float32, device=DEV),
             u=_rand(g, (T,)), u_next=_rand(g, (n,)), most=max(add))
    if own:
        from paper_2609_01024_b200 import binding as B
        s["verifier"] = B.DraftVerifier(max_seqs=n, max_path=max(add))
    return s


def _scores(q, k, scale, kvh, g):
    """scale q.k of one kv head: q [n, m, hq, d], k [n, l, hkv, d] -> [n, g, m, l]."""
    return torch.matmul(q[:, :, kvh * g:(kvh + 1) * g].permute(0, 2, 1, 3), k[:, :, kvh].transpose(1, 2).unsqueeze(1)).mul_(scale)


def _prepare_weigh(case, g, rng, dt):
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    ctx, add, kept = _ints(case["ctx"]), _ints(case["add"]), _ints(case["keep"])
    T, n = sum(add), len(ctx)
    count = kept if kept else add
    full = [c + m for c, m in zip(ctx, count)]
    pool = _Pool(g, rng, dt, 1, page, hkv, d, full, [max(1, x) for x in full])
    q = _randn(g, (T, hq, d), dt, 2.5)
    s = dict(T=T, n=n, pool=pool, seqs=_i32(np.arange(n)), cu=_cu(add), q=q, count=_i32(count), m_max=max(1, max(count)), l_max=max(1, max(full)), keep=None, n_keep=None)
    if kept:
        idx = np.full((n, max(1, max(kept))), -1, np.int32)
        for i, (a, m) in enumerate(zip(add, kept)):
            if m:
                idx[i, :m] = np.concatenate([[0], np.sort(1 + rng.permutation(a - 1)[:m - 1])])      # a branch of a tree
        s |= dict(keep=_i32(idx), n_keep=_i32(kept))
    # log sums of the counted rows, as the attention call has left them
    lse = torch.zeros((T, hq), dtype=torch.float32, device=DEV)
    rows, there, k, seen = _weigh_rows(s)
    lo = 0
    while lo < rows.shape[1]:                                            # pieces of rows, so that large prompts fit
        hi = min(rows.shape[1], lo + max(1, (1 << 28) // max(1, n * (hq // hkv) * s["l_max"])))
        qs = q[rows[:, lo:hi]].float()
        part = torch.stack([_scores(qs, k, d ** -0.5, h, hq // hkv).masked_fill_(~seen(lo, hi)[:, None], float("-inf")).logsumexp(-1) for h in range(hkv)], 1)
        part = part.permute(0, 3, 1, 2).reshape(n, hi - lo, hq)
        lse[rows[:, lo:hi][there[:, lo:hi]]] = part[there[:, lo:hi]]
        lo = hi
    s |= dict(lse=lse, saved=_rand(g, (n, pool.slots * page)) * 3, weight=torch.empty((n, pool.slots * page), device=DEV))
    if own:
        from paper_2609_01024_b200 import binding as B
        s["weights"] = B.CacheWeights(pool.handle, q_heads=hq, weight=s["weight"])
    return s


def _prepare_evict(case, g, rng, dt):
    hkv, d, page, layers = case["hkv"], case["d"], case["page"], case["layers"]
    lens, budget = _ints(case["lens"]), _ints(case["budget"])
    T, n = sum(lens), len(lens)
    pool = _Pool(g, rng, dt, layers, page, hkv, d, [0] * n, lens, values=False)
    # accumulated weights: heavy-tailed, a part of them exactly 0
    weight = torch.randn((n, pool.slots * page), generator=g, device=DEV).mul_(2).exp_()
    weight.masked_fill_(_rand(g, weight.shape) < 0.05, 0.0)
    s = dict(T=T, n=n, pool=pool, seqs=_i32(np.arange(n)), cu=_cu(lens), lens=_i32(lens), budget=_i32(budget), zero=_i32([0] * n), k=_randn(g, (layers, T, hkv, d), dt),
             v=_randn(g, (layers, T, hkv, d), dt), saved=weight, weight=torch.empty_like(weight))
    if own:
        from paper_2609_01024_b200 import binding as B
        s["weights"] = B.CacheWeights(pool.handle, q_heads=hkv, weight=s["weight"])
    return s


def prepare(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    f = {"rotate": _prepare_rotate, "verify": _prepare_verify, "weigh": _prepare_weigh, "evict": _prepare_evict}[case["op"]]
    return dict(f(case, g, rng, TYPES[case["dtype"]]), case=case, op=case["op"])


# --------------------------------------------------------------------------------------------------- plain forms

def _rows_of(cu, T):
    """Sequence and place inside it of every packed row."""
    t = torch.arange(T, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(cu[1:], t, right=True)
    return seq, t.long() - cu.long()[seq]


def _turn(x, weight, eps, cos, sin, rot, neighbours):
    """Norm and rotation of x [T, heads, d] in fp32."""
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * weight.float()
    r, rest = y[..., :rot], y[..., rot:]
    if neighbours:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([r, rest], -1).to(x.dtype)


def _plain_rotate(s):
    c = s["case"]
    angle = s["position"].double()[:, None, None] * s["inv_freq"]         # far positions: 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()
    s["q_out"].copy_(_turn(s["q"], s["q_weight"], s["eps"], cos, sin, c["rot"], c["pairs"] == "neighbours"))
    k = _turn(s["k"], s["k_weight"], s["eps"], cos, sin, c["rot"], c["pairs"] == "neighbours")
    out = dict(q=s["q_out"])
    if c["into"] != "cache":
        s["k_out"].copy_(k)
        out["k"] = s["k_out"]
    if c["into"] != "packed":
        pool = s["pool"]
        seq, at = _rows_of(s["cu"], s["T"])
        p = pool.len.long()[seq] - (s["cu"][1:] - s["cu"][:-1]).long()[seq] + at
        page = pool.table[seq, p // pool.page].long()
        pool.k[0][page, :, p % pool.page] = k
        pool.v[0][page, :, p % pool.page] = s["v"]
        out |= dict(k_pool=pool.k, v_pool=pool.v)
    return out


def _plain_verify(s):
    n, T = s["n"], s["T"]
    x = s["x"].double()                                                    # decisions and sums of many words: 64 bits
    x = torch.where(torch.isfinite(x), x, torch.full_like(x, float("-inf")))
    seq, at = _rows_of(s["cu"], T)
    t = s["temperature"].double()
    greedy = (t <= 0)[seq][:, None]
    p = torch.softmax(x / torch.where(t > 0, t, torch.ones_like(t))[seq][:, None], 1)
    p = torch.where(torch.isnan(p), torch.zeros_like(p), p)               # a row without an eligible word
    p = torch.where(greedy, torch.zeros_like(p).scatter_(1, x.argmax(1, keepdim=True), 1.0), p)
    first = s["cu"][:-1].long()
    size = (s["cu"][1:] - s["cu"][:-1]).long()
    cur = torch.zeros_like(first)
    r, R = p[first], torch.ones_like(t)
    path = torch.full((n, s["most"]), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = 0
    length = torch.ones_like(first)
    for j in range(1, s["most"]):
        row = torch.minimum(first + j, torch.full_like(first, T - 1))
        parent = s["parent"][row].long() if s["parent"] is not None else torch.full_like(first, j - 1)
        asked = (j < size) & (parent == cur)
        token = s["tokens"][row].long()[:, None]
        if s["near"] is not None:
            q = s["near"][first + cur].double()
        else:
            q = torch.zeros_like(r).scatter_(1, token, 1.0)
        taken = asked & (s["u"][row].double() * R * q.gather(1, token)[:, 0] < r.gather(1, token)[:, 0])
        left = (r - R[:, None] * q).clamp_(min=0)
        refused = asked & ~taken
        r = torch.where(taken[:, None], p[row], torch.where(refused[:, None], left, r))
        R = torch.where(taken, torch.ones_like(R), torch.where(refused, left.sum(1), R))
        gone = refused & (R <= 0)                                          # nothing left: the target's own again
        r = torch.where(gone[:, None], p[first + cur], r)
        R = torch.where(gone, torch.ones_like(R), R)
        cur = torch.where(taken, torch.full_like(cur, j), cur)
        length = length + taken
        path.scatter_(1, length[:, None] - 1, cur.int()[:, None])
    total = r.cumsum(1)
    nxt = (total <= s["u_next"].double()[:, None] * total[:, -1:]).sum(1)
    nxt = torch.where(total[:, -1] > 0, nxt, torch.full_like(nxt, -1))
    return dict(keep=path, n_keep=length.int(), next=nxt.int())


def _weigh_rows(s):
    """Packed row [n, m_max] of every counted row, whether there is one, the keys [n, l_max, hkv, d] in fp32, and which positions
    rows lo..hi see."""
    pool, n = s["pool"], s["n"]
    m = torch.arange(s["m_max"], device=DEV)[None, :].expand(n, -1)
    there = m < s["count"][:, None]
    rows = s["cu"][:-1].long()[:, None] + (m if s["keep"] is None else s["keep"][:, :s["m_max"]].long())
    rows = torch.where(there, rows, torch.zeros_like(rows))
    p = torch.arange(s["l_max"], device=DEV)
    pages = pool.table[:, p // pool.page].clamp(min=0).long()
    k = pool.k[0][pages, :, p % pool.page].float()
    base = (pool.len - s["count"]).long()

    def seen(lo, hi):
        return (p[None, None, :] <= (base[:, None] + m[:, lo:hi])[:, :, None]) & there[:, lo:hi, None]
    return rows, there, k, seen


def _plain_weigh(s):
    c, pool, n = s["case"], s["pool"], s["n"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    rows, there, k, seen = _weigh_rows(s)
    got = torch.zeros((n, s["l_max"]), device=DEV)
    q, lse = s["q"][rows].float(), s["lse"][rows]                          # [n, m, hq, d], [n, m, hq]
    hidden = ~seen(0, rows.shape[1])[:, None]
    for h in range(hkv):
        g = hq // hkv
        x = _scores(q, k, d ** -0.5, h, g).sub_(lse[:, :, h * g:(h + 1) * g].permute(0, 2, 1).unsqueeze(-1)).exp_()
        got += x.masked_fill_(hidden, 0.0).sum((1, 2))
    w = s["weight"].copy_(s["saved"])
    p = torch.arange(s["l_max"], device=DEV)[None, :]
    new = (p >= (pool.len - s["count"])[:, None]) & (p < pool.len[:, None])
    w[:, :s["l_max"]] = torch.where(p < pool.len[:, None], torch.where(new, torch.zeros_like(got), w[:, :s["l_max"]]) + got, w[:, :s["l_max"]])
    return dict(weight=w)


def _plain_evict(s):
    c, pool, n = s["case"], s["pool"], s["n"]
    page, pages, slots = pool.page, pool.pages, pool.slots
    # reserve: the lowest free pages in call order (nothing is in use)
    have = (s["lens"].long() + page - 1) // page
    at = torch.arange(slots, device=DEV)[None, :]
    first = have.cumsum(0) - have
    mine = at < have[:, None]
    table = torch.where(mine, first[:, None] + at, torch.full_like(at, -1).expand(n, -1))
    # write the prompts' rows
    seq, p = _rows_of(s["cu"], s["T"])
    where = table[seq, p // page]
    pool.k[:, where, :, p % page] = s["k"].permute(1, 0, 2, 3)
    pool.v[:, where, :, p % page] = s["v"].permute(1, 0, 2, 3)
    # what stays of each sequence: sinks, recent ones, and the heaviest, in order
    w = s["weight"].copy_(s["saved"])
    place = torch.arange(slots * page, device=DEV)[None, :]
    length, budget = s["lens"].long()[:, None], s["budget"].long()[:, None]
    inside = place < length
    safe = inside & ((place < c["sinks"]) | (place >= length - c["recent"]))
    key = torch.where(safe, torch.full_like(w, float("inf")), torch.where(inside, w, torch.full_like(w, float("-inf"))))
    order = torch.sort(key, dim=1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, place.expand(n, -1).contiguous())
    stays = inside & ((rank < budget) | (length <= budget))
    to = stays.long().cumsum(1) - 1
    left = torch.minimum(length, budget)[:, 0]
    # the place that every place's content comes from; those behind the budget keep theirs
    every = place.expand(n, -1).contiguous()
    source = torch.cat([every, every[:, :1]], 1).scatter_(1, torch.where(stays, to, torch.full_like(to, slots * page)), every)[:, :-1]
    w.copy_(torch.where(place < left[:, None], w.gather(1, source), w))
    pick = s["cu"].long()[seq] + source[seq, p]
    for x in (pool.k, pool.v):
        x[:, where, :, p % page] = x[:, where, :, p % page][pick]
    used = (left + page - 1) // page
    still = (at < used[:, None]) & mine
    ref = torch.zeros(pages + 1, dtype=torch.int32, device=DEV)
    ref[torch.where(still, table, torch.full_like(table, pages))] = 1
    ref = ref[:-1]
    after = torch.cat([left.int(), ref, torch.where(still, table, torch.full_like(table, -1)).int().reshape(-1)])
    pool.len.zero_()
    pool.ref.zero_()
    pool.table.fill_(-1)
    return dict(k=pool.k, v=pool.v, weight=w, after=after, book=pool.book)


# ----------------------------------------------------------------------------------------------- the user's calls

def _own_rotate(s):
    c, out = s["case"], dict(q=s["q_out"])
    if c["into"] == "packed":
        s["rotation"].rotate(s["q"], s["k"], s["position"], s["q_out"], s["k_out"])
    else:
        s["rotation"].rotate_cached(s["q"], s["k"], s["v"], s["position"], s["pool"].handle, 0, s["seqs"], s["cu"], s["q_out"], s["k_out"])
        out |= dict(k_pool=s["pool"].k, v_pool=s["pool"].v)
    if c["into"] != "cache":
        out["k"] = s["k_out"]
    return out


def _own_verify(s):
    keep, n_keep, nxt = s["verifier"].verify(s["x"], s["tokens"], s["cu"], s["u"], s["u_next"], parent=s["parent"], draft_probs=s["near"], temperature=s["temperature"])
    return dict(keep=keep, n_keep=n_keep, next=nxt)


def _own_weigh(s):
    s["weight"].copy_(s["saved"])
    s["weights"].add(s["q"], s["lse"], 0, s["seqs"], s["cu"], keep=s["keep"], n_keep=s["n_keep"], fresh=True)
    return dict(weight=s["weight"])


def _own_evict(s):
    c, cache = s["case"], s["pool"].handle
    cache.reserve(s["seqs"], s["lens"])
    cache.write(s["k"], s["v"], s["seqs"], s["cu"])
    s["weight"].copy_(s["saved"])
    s["weights"].evict(s["seqs"], s["budget"], sinks=c["sinks"], recent=c["recent"])
    after = s["pool"].book.clone()
    cache.trim(s["seqs"], s["zero"])
    return dict(k=cache.k, v=cache.v, weight=s["weight"], after=after, book=s["pool"].book)


def run(s):
    op = s["op"]
    if own:
        return {"rotate": _own_rotate, "verify": _own_verify, "weigh": _own_weigh, "evict": _own_evict}[op](s)
    return {"rotate": _plain_rotate, "verify": _plain_verify, "weigh": _plain_weigh, "evict": _plain_evict}[op](s)


# ------------------------------------------------------------------------------------------------------- the work

def work(case):
    op, e = case["op"], 2 if case["dtype"] == "bf16" else 4
    if op == "rotate":
        T, hq, hkv, d = sum(_ints(case["add"])), case["hq"], case["hkv"], case["d"]
        rows = 2 * hq + 2 * hkv if case["into"] == "packed" else 2 * hq + 4 * hkv if case["into"] == "cache" else 2 * hq + 5 * hkv
        return dict(bytes=e * T * d * rows + 4 * T, flops=8 * T * d * (hq + hkv))
    if op == "verify":
        # rows that the walk must read: three of four drafts are taken in a chain, a branch of about three in a tree; a refusal
        # costs the drafter's row too
        rows = words = 0.0
        for a in _ints(case["add"]):
            seen = min(3.0, 1 + 0.3 * (a - 1)) if case["tree"] else sum(0.75 ** k for k in range(a))
            rows += seen
            words += (1 - 0.75 ** (a - 1)) if case["drafts"] else 0.0
        return dict(bytes=int(case["vocab"] * (e * rows + 4 * words)), flops=int(4 * case["vocab"] * rows))
    if op == "weigh":
        ctx, add, kept = _ints(case["ctx"]), _ints(case["add"]), _ints(case["keep"])
        count = kept if kept else add
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        live = [c + m if m else 0 for c, m in zip(ctx, count)]
        seen = sum(m * c + m * (m + 1) // 2 for c, m in zip(ctx, count))
        return dict(bytes=e * hkv * d * sum(live) + e * hq * d * sum(count) + 4 * hq * sum(count) + 8 * sum(live), flops=2 * d * hq * seen)
    lens, budget = _ints(case["lens"]), _ints(case["budget"])
    row = 2 * e * case["hkv"] * case["d"] * case["layers"]                 # K and V of a token in all layers
    moved = sum(max(0, b - case["sinks"]) for x, b in zip(lens, budget) if b < x)
    return dict(bytes=2 * row * (sum(lens) + moved) + 4 * sum(lens), flops=0)


# ------------------------------------------------------------------------------------------ the definition, 64 bits

def _exact_rotate(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    angle = s["position"].double()[:, None] * s["inv_freq"][None, :]
    z = torch.polar(torch.ones_like(angle), angle)[:, None, :]            # rotation as a complex product

    def one(x, weight):
        y = x.double().clone()
        if weight is not None:
            y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / c["d"] + s["eps"]) * weight.double()
        if half:
            even, odd = (slice(0, rot, 2), slice(1, rot, 2)) if c["pairs"] == "neighbours" else (slice(0, half), slice(half, rot))
            w = torch.complex(y[..., even], y[..., odd]) * z
            y[..., even], y[..., odd] = w.real, w.imag
        return y
    q, k = one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])
    out = dict(q=q)
    if c["into"] != "cache":
        out["k"] = k
    if c["into"] != "packed":
        pool = s["pool"]
        kp, vp = pool.k.double(), pool.v.double()
        table = pool.table.cpu().numpy()
        a = 0
        for i, (past, n) in enumerate(zip(_ints(c["ctx"]), _ints(c["add"]))):
            for slot in range(past // pool.page, _pages_of(past + n, pool.page) if n else 0):
                lo, hi = max(past, slot * pool.page), min(past + n, (slot + 1) * pool.page)
                rows, to = slice(a + lo - past, a + hi - past), slice(lo - slot * pool.page, hi - slot * pool.page)
                kp[0, int(table[i, slot]), :, to] = k[rows].transpose(0, 1)
                vp[0, int(table[i, slot]), :, to] = s["v"][rows].double().transpose(0, 1)
            a += n
        out |= dict(k_pool=kp, v_pool=vp)
    return out


def _exact_verify(s):
    add = _ints(s["case"]["add"])
    tokens, u, u_next, temp = (s[x].cpu().numpy() for x in ("tokens", "u", "u_next", "temperature"))
    parent = None if s["parent"] is None else s["parent"].cpu().numpy()
    keep = np.full((s["n"], s["most"]), -1, np.int32)
    n_keep, nxt = np.zeros(s["n"], np.int32), np.zeros(s["n"], np.int32)

    def target(row, t):
        x = s["x"][row].double().cpu().numpy()
        ok = np.isfinite(x)
        if not ok.any():
            return np.zeros_like(x)
        x = np.where(ok, x, -np.inf)
        if t <= 0:
            return (np.arange(len(x)) == int(np.argmax(x))).astype(np.float64)
        w = np.exp((x - x.max()) / float(t))
        return w / w.sum()
    a = 0
    for i, n in enumerate(add):
        path, p = [0], target(a, temp[i])
        r = p.copy()
        while True:
            for j in range(path[-1] + 1, n):
                if (j - 1 if parent is None else int(parent[a + j])) != path[-1]:
                    continue
                x, mass = int(tokens[a + j]), r.sum()
                q = s["near"][a + path[-1]].double().cpu().numpy() if s["near"] is not None else (np.arange(len(r)) == x).astype(np.float64)
                if float(u[a + j]) * q[x] < r[x] / mass:
                    path.append(j)
                    break
                r = np.maximum(r / mass - q, 0)
                if not r.sum() > 0:
                    r = p.copy()
            else:
                break
            p = target(a + path[-1], temp[i])
            r = p.copy()
        total = np.cumsum(r)
        keep[i, :len(path)], n_keep[i] = path, len(path)
        nxt[i] = int(np.searchsorted(total, float(u_next[i]) * total[-1], side="right")) if total[-1] > 0 else -1
        a += n
    return dict(keep=torch.tensor(keep, device=DEV), n_keep=torch.tensor(n_keep, device=DEV), next=torch.tensor(nxt, device=DEV))


def _exact_weigh(s):
    c, pool = s["case"], s["pool"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    g = hq // hkv
    w = s["saved"].double()
    table = pool.table.cpu().numpy()
    a = 0
    for i, (past, n) in enumerate(zip(_ints(c["ctx"]), _ints(c["add"]))):
        mine = list(range(n)) if s["keep"] is None else [int(x) for x in s["keep"][i, :int(s["n_keep"][i])]]
        m = len(mine)
        w[i, past:past + m] = 0
        if m:
            pages = torch.tensor(table[i, :_pages_of(past + m, pool.page)].astype(np.int64), device=DEV)
            k = pool.k[0, pages].transpose(1, 2).reshape(-1, hkv, d)[:past + m].double()
            rows = torch.tensor(mine, device=DEV) + a
            for lo in range(0, m, 1024):
                pick = rows[lo:lo + 1024]
                l = past + min(m, lo + 1024)                              # nobody here sees more
                hidden = torch.arange(l, device=DEV)[None, :] > past + lo + torch.arange(len(pick), device=DEV)[:, None]
                for h in range(hq):
                    x = (s["q"][pick, h].double() @ k[:l, h // g].T) * d ** -0.5 - s["lse"][pick, h].double()[:, None]
                    w[i, :l] += x.masked_fill_(hidden, float("-inf")).exp_().sum(0)
        a += n
    return dict(weight=w)


def _exact_evict(s):
    c, pool = s["case"], s["pool"]
    page = pool.page
    k, v = pool.k.double(), pool.v.double()
    w = s["saved"].double().cpu().numpy().copy()
    lens, budget = _ints(c["lens"]), _ints(c["budget"])
    table = np.full((s["n"], pool.slots), -1, np.int32)
    ref = np.zeros(pool.pages, np.int32)
    left, page_at, a = [], 0, 0
    for i, (n, b) in enumerate(zip(lens, budget)):
        m = _pages_of(n, page)
        ids = np.arange(page_at, page_at + m)
        page_at += m
        order = np.arange(n)
        if n > b:
            free = [p for p in range(n) if c["sinks"] <= p < n - c["recent"]]
            many = b - (n - len(free))
            heavy = sorted(free, key=lambda p: (-w[i, p], p))[:many]
            order = np.array(sorted(set(range(n)) - (set(free) - set(heavy))), dtype=np.int64)
        rows = np.concatenate([order, np.arange(len(order), n)])          # row of the prompt that each place ends with
        for x, y in ((k, s["k"]), (v, s["v"])):
            block = y[:, torch.tensor(a + rows, device=DEV)].double().transpose(1, 2)            # [layers, hkv, n, d]
            for j in range(m):
                part = block[:, :, j * page:(j + 1) * page]
                x[:, int(ids[j]), :, :part.shape[2]] = part
        w[i, :len(order)] = w[i, order]
        left.append(len(order))
        used = _pages_of(len(order), page)
        table[i, :used], ref[ids[:used]] = ids[:used], 1
        a += n
    book = np.concatenate([np.zeros(s["n"] + pool.pages, np.int32), np.full(table.size, -1, np.int32)])
    return dict(k=k, v=v, weight=torch.tensor(w, device=DEV), after=_i32(np.concatenate([np.asarray(left), ref, table.reshape(-1)])), book=_i32(book))


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "verify": _exact_verify, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](s)
