"""Attention over packed prompts and over the paged cache against the 64-bit definition.

Bounds, derived from the arithmetic and element by element.  With A = sum a_p |v_p| / sum a_p (the reference returns it):
bf16 (8 significant bits: rounding to nearest is off by up to u = eps / 2 = 2^-8 of the value): every weight is rounded and the
result once more: |do| <= u A + u |o|, and the fp32 scores
(products exact, at most 128 of them summed, relative 2^-24 each, sizes of some tens) and exponentials move a weight by less
than 3e-4 of itself.  fp32: the scores' error d * 2^-24 * sum |q k| * scale stays under 1e-4 for these inputs, and so does
everything after it.  lse is an fp32 number of size ~10 with the scores' error: 1e-4."""
import numpy as np
import pytest
import torch

import serving_reference as R
from paper_2609_01024_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (B.PCOMOE_BF16, torch.bfloat16), "f32": (B.PCOMOE_FP32, torch.float32)}


def check(out, lse, ref, dtype):
    o, want_lse, size = ref
    out, lse = out.double().cpu(), lse.double().cpu()
    assert torch.equal(torch.isnan(out), torch.isnan(o))
    u = torch.finfo(torch.bfloat16).eps / 2
    bound = (u + 3e-4) * size + u * o.abs() if dtype == "bf16" else 1e-4 * size
    bad = ((out - o).abs() > bound + 1e-30) & ~torch.isnan(o)
    assert not bad.any(), (int(bad.sum()), float((out - o).abs()[bad].max()))
    fine = torch.isfinite(want_lse)
    assert torch.equal(lse[~fine].isnan(), want_lse[~fine].isnan())
    assert torch.equal(lse[torch.isinf(want_lse)], want_lse[torch.isinf(want_lse)])
    assert ((lse - want_lse)[fine].abs() <= 1e-4).all()


def randn(seed, *shape, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def ints(v):
    return torch.tensor(np.asarray(v, np.int32), device=DEV)


def cu_of(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]))


def make(dtype, hq, hkv, d, T, n, scale=None):
    return B.Attention(q_heads=hq, kv_heads=hkv, head_dim=d, max_tokens=T, max_seqs=n, dtype=TYPES[dtype][0], scale=scale, device=DEV)


PROMPTS = [[1], [2, 0, 1], [63, 64, 65, 1], [128, 129, 127], [300, 0, 0, 5], [257], [1] * 70]


@pytest.mark.parametrize("lens", PROMPTS, ids=str)
@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (3, 1), (14, 2)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt(dtype, d, heads, lens):
    hq, hkv = heads
    T, dt = sum(lens), TYPES[dtype][1]
    qkv = randn(len(lens) + d, T, (hq + 2 * hkv) * d, dtype=dt, std=1.2)
    x = qkv.to(DEV)
    parts = lambda y: (y[:, :hq * d].unflatten(1, (hq, d)), y[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)),
                       y[:, (hq + hkv) * d:].unflatten(1, (hkv, d)))
    at = make(dtype, hq, hkv, d, T, len(lens))
    out, lse = at.prompt(*parts(x), cu_of(lens))
    assert at.device_status() == 0
    check(out, lse, R.prompt(*parts(qkv), lens, d ** -0.5), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_longer_than_many_tiles(dtype):
    """Several tiles of rows and of keys, a scale of its own, an output with a wider row."""
    hq, hkv, d, lens = 4, 2, 128, [900, 531]
    T, dt = sum(lens), TYPES[dtype][1]
    q, k, v = (randn(i, T, h, d, dtype=dt) for i, h in enumerate((hq, hkv, hkv)))
    wide = torch.full((T, hq * d + 64), 7.0, dtype=dt, device=DEV)
    lse = torch.zeros(T, hq, device=DEV)
    at = make(dtype, hq, hkv, d, T, 2, scale=0.2)
    at.prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_of(lens), out=wide[:, :hq * d].unflatten(1, (hq, d)), lse=lse)
    check(wide[:, :hq * d].unflatten(1, (hq, d)), lse, R.prompt(q, k, v, lens, 0.2), dtype)
    assert bool((wide[:, hq * d:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_values_nobody_sees_do_not_matter(dtype):
    """NaN and infinities in later rows and in other sequences reach only the rows that see them."""
    hq, hkv, d, lens = 4, 2, 64, [70, 200, 33]
    T, dt = sum(lens), TYPES[dtype][1]
    q, k, v = (randn(i, T, h, d, dtype=dt) for i, h in enumerate((hq, hkv, hkv)))
    v[70 + 150, 0, 3] = float("nan")
    v[70 + 160, 1, 5] = float("inf")
    k[70 + 170, 1] = float("nan")
    at = make(dtype, hq, hkv, d, T, 3)
    out, lse = at.prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_of(lens))
    o, want, size = R.prompt(q, k, v, lens, d ** -0.5)
    free = torch.isfinite(o).all(-1) & torch.isfinite(want)                      # heads and rows without such a value in sight
    assert free[:70].all() and free[270:].all() and free[70:220].all() and not free[269].any()
    out, lse = out.double().cpu(), lse.double().cpu()
    assert torch.isfinite(out[free]).all()
    check(out[free], lse[free], (o[free], want[free], size[free]), dtype)
    assert torch.isnan(out[220:240, 0, 3]).all() and torch.isnan(out[240:270, 2:]).all()
    assert torch.isinf(out[230:240, 2, 5]).all()


def test_prompt_rows_past_the_last_sequence_are_not_written():
    at = make("bf16", 2, 1, 64, 40, 2)
    at.out.fill_(3.0)
    q, k, v = (randn(i, 40, h, 64, dtype=torch.bfloat16).to(DEV) for i, h in enumerate((2, 1, 1)))
    out, _ = at.prompt(q, k, v, cu_of([9, 8]))
    assert bool((out[17:] == 3.0).all()) and not bool((out[:17] == 3.0).any())
    assert at.device_status() == 0


def test_prompt_bad_lengths_are_reported_and_skipped():
    at = make("bf16", 2, 1, 64, 40, 3)
    q, k, v = (randn(i, 40, h, 64, dtype=torch.bfloat16).to(DEV) for i, h in enumerate((2, 1, 1)))
    at.out.fill_(3.0)
    out, _ = at.prompt(q, k, v, ints([0, 10, 5, 50]))
    assert at.device_status() == 7
    assert bool((out[10:] == 3.0).all()) and not bool((out[:10] == 3.0).any())
    assert at.device_status() == 0                                                # the word is cleared once read


# ------------------------------------------------------------------------------------------------- over the cache

def fill_cache(dtype, hkv, d, page, lens, seed, layers=2, spare=3, poison=True):
    """A cache whose pages are shuffled; every row outside the sequences is NaN (stale memory)."""
    pages = sum(-(-n // page) for n in lens) + spare
    c = B.PagedCache(layers=layers, pages=pages, page_size=page, kv_heads=hkv, head_dim=d, max_seqs=len(lens),
                     max_pages=max(1, max(-(-n // page) for n in lens)), dtype=TYPES[dtype][0], device=DEV)
    if poison:
        c.k.fill_(float("nan")), c.v.fill_(float("nan"))
    order = np.random.default_rng(seed).permutation(pages)
    table = np.full((len(lens), c.c.max_pages), -1, np.int32)
    keys, values, at = [], [], 0
    for s, n in enumerate(lens):
        kk, vv = (randn(seed * 100 + 2 * s + i, n, hkv, d, dtype=TYPES[dtype][1]) for i in (0, 1))
        for p in range(n):
            if p % page == 0:
                table[s, p // page] = order[at]
                at += 1
        for slot in range(-(-n // page)):
            m = min(page, n - slot * page)
            for pool, x in ((c.k, kk), (c.v, vv)):
                pool[1, int(table[s, slot]), :, :m] = x[slot * page:slot * page + m].transpose(0, 1).to(DEV)
        keys.append(kk), values.append(vv)
    c.seq_len.copy_(ints(lens))
    c.page_table.copy_(ints(table))
    ref = np.zeros(pages, np.int32)
    ref[table[table >= 0]] = 1
    c.page_ref.copy_(ints(ref))
    return c, keys, values


def seen_of(length, n, tree):
    see = np.ones((n, length), bool)
    see[:, length - n:] = np.tril(np.ones((n, n), bool)) if tree is None else tree
    return torch.from_numpy(see)


CACHED = [  # contexts, new tokens
    ([0], [1]), ([1, 0, 15], [1, 1, 1]), ([63, 64, 65, 200], [1, 1, 1, 1]), ([500, 3], [1, 1]),
    ([0, 40, 129], [3, 1, 7]), ([100, 17, 64, 255], [33, 5, 64, 1]), ([700], [130]), ([31, 0], [0, 20])]


@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("lens", CACHED, ids=str)
@pytest.mark.parametrize("shape", [(8, 8, 64, 16), (8, 2, 128, 32), (7, 1, 128, 64), (16, 2, 64, 128)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached(dtype, shape, lens, tree):
    hq, hkv, d, page = shape
    ctx, add = lens
    full = [c + a for c, a in zip(ctx, add)]
    cache, keys, values = fill_cache(dtype, hkv, d, page, full, seed=3)
    T = sum(add)
    q = randn(9, T, hq, d, dtype=TYPES[dtype][1], std=1.2)
    rng = np.random.default_rng(5)
    trees = [R.tree_bits(rng, n) if tree else None for n in add]
    words = (max(add) + 31) // 32 + 1                                             # one word more than needed
    mask = R.pack_bits(trees, words).to(DEV) if tree else None
    at = make(dtype, hq, hkv, d, T, len(ctx))
    out, lse = at.cached(q.to(DEV), cache, 1, ints(range(len(ctx))), cu_of(add), mask)
    assert at.device_status() == 0
    see = [seen_of(n, a, t) for n, a, t in zip(full, add, trees)]
    check(out, lse, R.cached(q, keys, values, add, see, d ** -0.5), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("counts", [[1, 1], [24, 40]], ids=str)
def test_cached_long_context_is_cut_and_joined(dtype, counts):
    """Contexts of thousands of tokens on few heads: many blocks of the grid share one tile."""
    hq, hkv, d, page = 4, 1, 128, 64
    full = [5000 + counts[0], 2111 + counts[1]]
    cache, keys, values = fill_cache(dtype, hkv, d, page, full, seed=4)
    q = randn(2, sum(counts), hq, d, dtype=TYPES[dtype][1], std=1.2)
    at = make(dtype, hq, hkv, d, sum(counts), 2)
    ref = R.cached(q, keys, values, counts, [seen_of(n, a, None) for n, a in zip(full, counts)], d ** -0.5)
    first = None
    for _ in range(3):                                                            # counters are left at zero; bits repeat
        out, lse = at.cached(q.to(DEV), cache, 1, ints([0, 1]), cu_of(counts))
        check(out, lse, ref, dtype)
        if first is None:
            first = (out.clone(), lse.clone())
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.parametrize("n", [4, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_masked_drafts_do_not_matter(dtype, n):
    """NaN and infinities in drafted tokens reach only the rows whose mask names them; a row that sees nothing is 0, -inf."""
    hq, hkv, d, page = 4, 2, 64, 16
    cache, keys, values = fill_cache(dtype, hkv, d, page, [n, 50 + n], seed=6)
    rng = np.random.default_rng(1)
    trees = [R.tree_bits(rng, n) for _ in range(2)]
    trees[0][0, :] = False                                                        # sees nothing: no context, no bit
    trees[0][:, 2] = False
    trees[1][:, 1] = False
    for s, at_token in ((0, 2), (1, 51)):
        slot, r = int(cache.page_table[s, at_token // page]), at_token % page
        for pool, host in ((cache.k, keys), (cache.v, values)):
            pool[1, slot, :, r] = float("nan")
            host[s][at_token] = float("nan")
    q = randn(8, 2 * n, hq, d, dtype=TYPES[dtype][1])
    at = make(dtype, hq, hkv, d, 2 * n, 2)
    out, lse = at.cached(q.to(DEV), cache, 1, ints([0, 1]), cu_of([n, n]), R.pack_bits(trees, 2).to(DEV))
    see = [seen_of(n, n, trees[0]), seen_of(50 + n, n, trees[1])]
    ref = R.cached(q, keys, values, [n, n], see, d ** -0.5)
    assert torch.isfinite(out).all()
    assert bool((out[0] == 0).all()) and bool((lse[0] == float("-inf")).all())
    check(out, lse, ref, dtype)


def test_cached_one_sequence_for_many_groups():
    """The same sequence named twice: its queries are then the last tokens of both groups."""
    cache, keys, values = fill_cache("bf16", 2, 64, 16, [90], seed=7)
    q = randn(3, 2, 4, 64, dtype=torch.bfloat16)
    at = make("bf16", 4, 2, 64, 2, 2)
    out, lse = at.cached(q.to(DEV), cache, 1, ints([0, 0]), cu_of([1, 1]))
    check(out, lse, R.cached(q, keys * 2, values * 2, [1, 1], [seen_of(90, 1, None)] * 2, 0.125), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_device_errors(dtype):
    cache, keys, values = fill_cache(dtype, 2, 64, 16, [30, 5, 12], seed=8)
    q = randn(3, 9, 4, 64, dtype=TYPES[dtype][1]).to(DEV)
    at = make(dtype, 4, 2, 64, 9, 3)
    ref = R.cached(q.cpu()[:1], keys[:1], values[:1], [1], [seen_of(30, 1, None)], 0.125)
    for seqs, counts in (([0, 7, 2], [1, 1, 1]), ([0, -1, 2], [1, 1, 1]), ([0, 1, 2], [1, 6, 1])):   # no such sequence; longer than cached
        out, lse = at.cached(q[:sum(counts)], cache, 1, ints(seqs), cu_of(counts))
        assert at.device_status() == 7
        check(out[:1], lse[:1], ref, dtype)
        n = counts[1]
        assert bool((out[1:1 + n] == 0).all()) and bool((lse[1:1 + n] == float("-inf")).all())
    out, lse = at.cached(q[:1], cache, 1, ints([0]), cu_of([1]))
    assert at.device_status() == 0


def test_on_another_stream_and_in_a_graph():
    """The calls follow the current stream; a captured step reruns on whatever the tensors hold by then."""
    cache, keys, values = fill_cache("bf16", 2, 128, 32, [200, 77], seed=9)
    q = randn(1, 2, 8, 128, dtype=torch.bfloat16).to(DEV)
    at = make("bf16", 8, 2, 128, 2, 2)
    seqs, cu = ints([0, 1]), cu_of([1, 1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        at.cached(q, cache, 1, seqs, cu)
    s.synchronize()
    see = [seen_of(200, 1, None), seen_of(77, 1, None)]
    check(at.out[:2], at.lse[:2], R.cached(q.cpu(), keys, values, [1, 1], see, 128 ** -0.5), "bf16")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        at.cached(q, cache, 1, seqs, cu)
    q.copy_(randn(2, 2, 8, 128, dtype=torch.bfloat16))
    cache.seq_len.copy_(ints([150, 70]))
    g.replay()
    torch.cuda.synchronize()
    check(at.out[:2], at.lse[:2], R.cached(q.cpu(), [keys[0][:150], keys[1][:70]], [values[0][:150], values[1][:70]], [1, 1],
                                           [seen_of(150, 1, None), seen_of(70, 1, None)], 128 ** -0.5), "bf16")


def test_refusals():
    lib = B.load_library()
    at = make("bf16", 4, 2, 64, 8, 2)
    cache, _, _ = fill_cache("bf16", 2, 64, 16, [8, 8], seed=1)
    x = torch.zeros(8, 8, 64, dtype=torch.bfloat16, device=DEV)
    cu = cu_of([4, 4])
    p, stream = x.data_ptr(), None

    def prompt(cfg=at._cfg, T=8, n=2, c=cu.data_ptr(), q=p, qs=512, k=p, ks=512, v=p, vs=512, o=p, os=512, ws=at._ws):
        return lib.pcomoe_attn_prompt(cfg, T, n, c, q, qs, k, ks, v, vs, o, os, None, *ws, stream)

    assert prompt(T=0) == 0
    assert prompt(T=-1) == 2 and prompt(n=0) == 1 and prompt(c=None) == 1 and prompt(q=None) == 1 and prompt(k=None) == 1
    assert prompt(qs=255) == 1 and prompt(ks=127) == 1 and prompt(os=0) == 1                     # rows would overlap
    assert prompt(q=p + 2) == 4 and prompt(v=p + 8) == 4 and prompt(vs=516) == 4                 # 16-byte rule
    assert prompt(ws=(at._ws[0], at._ws[1] - 1)) == 3 and prompt(ws=(at._ws[0] + 4, at._ws[1])) == 3 and prompt(ws=(None, 0)) == 3
    import ctypes
    for field, value, status in (("head_dim", 96, 4), ("q_heads", 5, 1), ("kv_heads", 0, 1), ("dtype", 3, 1), ("scale", float("inf"), 1),
                                 ("struct_size", 8, 1)):
        cfg = B.pcomoe_attn_config.from_buffer_copy(at.cfg)
        setattr(cfg, field, value)
        assert prompt(cfg=ctypes.byref(cfg)) == status, field

    def cached(layer=0, T=8, n=2, seqs=cu.data_ptr(), mask=None, words=0, c=cache._ref, cfg=at._cfg):
        return lib.pcomoe_attn_cached(cfg, c, layer, T, n, seqs, cu.data_ptr(), p, 512, mask, words, p, 512, None, *at._ws, stream)

    assert cached(layer=2) == 1 and cached(layer=-1) == 1 and cached(seqs=None) == 1 and cached(c=None) == 1
    assert cached(words=9) == 2 and cached(words=-1) == 2 and cached(mask=p, words=0) == 1 and cached(T=-2) == 2 and cached(T=0) == 0
    other = B.pcomoe_attn_config.from_buffer_copy(at.cfg)
    other.kv_heads = 4
    assert cached(cfg=ctypes.byref(other)) == 1                                                  # not the cache's heads
    torch.cuda.synchronize()
    assert at.device_status() == 0
