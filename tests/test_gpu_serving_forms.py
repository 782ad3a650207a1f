"""Both sides of every rule by which the serving kernels choose their form (rows per sequence, tiles per SM, rows and words of
the logits), against the 64-bit definitions and with the bounds of the operators' own tests."""
import numpy as np
import pytest
import torch

import serving_reference as R
from test_gpu_attention import DEV, TYPES, check as check_attention, cu_of, fill_cache, ints, make, randn, seen_of
from test_gpu_scores import check as check_scores, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,V,top,dtype", [
    (2500, 300, 5, "bf16"), (2500, 300, 9, "bf16"), (2500, 1900, 8, "f32"),        # a warp per row, or teams where many are wanted
    (3600, 229, 32, "bf16"), (3600, 2600, 3, "f32"),                               # teams of two warps
    (700, 4200, 9, "bf16"), (700, 150, 32, "f32"),                                 # of four
    (300, 33000, 4, "f32"), (20, 33000, 32, "f32"), (2, 40001, 7, "bf16"),         # clusters
    (200, 7000, 32, "bf16"), (200, 260, 20, "bf16")])                              # a block per row
def test_scores(T, V, top, dtype):
    x = logits(T + V, T, V, dtype, std=2.0)
    x[torch.rand(T, V, generator=torch.Generator().manual_seed(1)) < 0.3] = float("-inf")
    x[1] = x[1].round()                                                            # equal words
    x[T // 2, 3:] = float("-inf")                                                  # fewer eligible words than ranks
    check_scores(x, [(11 * t) % V for t in range(T)], top)


@pytest.mark.parametrize("heads,lens", [((2, 1), [1000, 3]), ((3, 1), [700, 129]), ((6, 2), [43, 0, 86, 600]), ((16, 16), [520, 130]),
                                        ((2, 2), [5] * 140 + [300, 7])], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_tiles(dtype, heads, lens):
    """Few tiles (half as high, or a quarter in fp32) and many, groups that do and do not divide a tile, more than 128 sequences."""
    (hq, hkv), d, T = heads, 64, sum(lens)
    q, k, v = (randn(i, T, h, d, dtype=TYPES[dtype][1], std=1.2) for i, h in enumerate((hq, hkv, hkv)))
    at = make(dtype, hq, hkv, d, T, len(lens))
    out, lse = at.prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_of(lens))
    assert at.device_status() == 0
    check_attention(out, lse, R.prompt(q, k, v, lens, d ** -0.5), dtype)


@pytest.mark.parametrize("ctx,add", [
    ([90] * 5, [3] * 5), ([90] * 5, [4] * 5), ([90] * 5, [5] * 5),                 # 24, 32 and 40 rows per sequence and kv head
    ([5, 0, 300, 17, 60] * 8, [1, 2, 1, 4, 1] * 8),                                # more than 32 sequences, tiles not cut
    ([5, 0, 300, 17, 1500] * 8, [1, 30, 1, 17, 9] * 8),                            # more than 32 sequences, cut
    ([10, 100] * 60, [20, 40] * 60),                                               # more tiles than blocks of threads
    ([600, 20], [2, 6]), ([900], [9])], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_shares(dtype, ctx, add):
    hq, hkv, d, page = 16, 2, 64, 16
    full, T = [c + a for c, a in zip(ctx, add)], sum(add)
    cache, keys, values = fill_cache(dtype, hkv, d, page, full, seed=8)
    q = randn(4, T, hq, d, dtype=TYPES[dtype][1], std=1.2)
    rng = np.random.default_rng(2)
    trees = [R.tree_bits(rng, n) for n in add]
    at = make(dtype, hq, hkv, d, T, len(ctx))
    out, lse = at.cached(q.to(DEV), cache, 1, ints(range(len(ctx))), cu_of(add), R.pack_bits(trees, 2).to(DEV))
    assert at.device_status() == 0
    check_attention(out, lse, R.cached(q, keys, values, add, [seen_of(n, a, t) for n, a, t in zip(full, add, trees)], d ** -0.5), dtype)


@pytest.mark.parametrize("n", [7, 12, 20, 40])
def test_cached_values_nobody_sees_fp32_rest_tiles(n):
    """A tile's last rows worked on 16, 32 or 64 at a time; a NaN in one draft's value reaches the rows that see it."""
    hq, hkv, d, page = 4, 2, 128, 32
    cache, keys, values = fill_cache("f32", hkv, d, page, [70 + n], seed=9)
    tree = R.tree_bits(np.random.default_rng(3), n)
    tree[:, 3], tree[n - 1, 3] = False, True
    slot, r = int(cache.page_table[0, 73 // page]), 73 % page
    cache.v[1, slot, :, r, 5] = float("nan")
    values[0][73, :, 5] = float("nan")
    q = randn(6, n, hq, d, dtype=torch.float32)
    at = make("f32", hq, hkv, d, n, 1)
    out, lse = at.cached(q.to(DEV), cache, 1, ints([0]), cu_of([n]), R.pack_bits([tree], 2).to(DEV))
    assert torch.isfinite(out[:n - 1]).all() and torch.isnan(out[n - 1, :, 5]).all()
    check_attention(out, lse, R.cached(q, keys, values, [n], [seen_of(70 + n, n, tree)], d ** -0.5), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_nan_is_not_hidden(dtype):
    """A NaN in a query, and in a first key, which is all that its own row sees, gives NaN there and nowhere else."""
    hq, hkv, d, lens = 4, 2, 64, [150, 1, 20]
    T = sum(lens)
    q, k, v = (randn(i, T, h, d, dtype=TYPES[dtype][1], std=1.2) for i, h in enumerate((hq, hkv, hkv)))
    q[7, 1, 3] = q[149, 2, 0] = q[165, 0, 9] = float("nan")
    k[150, 0, 5] = float("nan")
    at = make(dtype, hq, hkv, d, T, len(lens))
    out, lse = at.prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_of(lens))
    ref = R.prompt(q, k, v, lens, d ** -0.5)
    assert torch.isnan(ref[0][7, 1]).all() and torch.isnan(ref[0][150, :2]).all() and torch.isfinite(ref[0][150, 2:]).all()
    check_attention(out, lse, ref, dtype)


@pytest.mark.parametrize("ctx,add", [([50, 0], [2, 1]), ([60, 9], [40, 17]), ([4000, 30], [2, 2]), ([4000, 30], [40, 40])], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_nan_is_not_hidden(dtype, ctx, add):
    """The same over the cache, where a tile may be whole or cut into many parts."""
    hq, hkv, d, page = 4, 1, 64, 64
    full, T = [c + a for c, a in zip(ctx, add)], sum(add)
    cache, keys, values = fill_cache(dtype, hkv, d, page, full, seed=5)
    q = randn(3, T, hq, d, dtype=TYPES[dtype][1], std=1.2)
    q[0, 1, 3] = q[T - 1, 0, 63] = float("nan")
    at = make(dtype, hq, hkv, d, T, len(ctx))
    out, lse = at.cached(q.to(DEV), cache, 1, ints(range(len(ctx))), cu_of(add))
    ref = R.cached(q, keys, values, add, [seen_of(n, a, None) for n, a in zip(full, add)], d ** -0.5)
    assert int(torch.isnan(ref[1]).sum()) == 2
    check_attention(out, lse, ref, dtype)
