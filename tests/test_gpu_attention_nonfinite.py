"""NaN and infinities in values: what a row sees counts however small its weight, what it does not see never does.

One key scores 100 above the others, so that the others' weights (e^-100 = 2^-144) are zero in fp32 and not in the 64-bit
definition: a NaN among their values has to come out, wherever a block of keys is masked or a tile is cut.  The bounds are those of
test_gpu_attention; lse is then a number of size 100 behind five roundings of 2^-24 (scale times log2 e, the product with the
score, ln 2, the product with it, the sum): 100 * 5 * 2^-24 = 3e-5, inside the 1e-4 that `check` allows."""
import numpy as np
import pytest
import torch

import serving_reference as R
from test_gpu_attention import DEV, TYPES, check, cu_of, fill_cache, ints, make, randn, seen_of

pytestmark = pytest.mark.gpu
SCALE = 0.125


def far_apart(q, k, high):
    """Every row's score with key `high` becomes 100 (32 * 25 / 8), with the others about 0."""
    q[..., 0] = 32.0
    k[:, :, 0] = 0.0
    k[:, :, 1:] *= 0.25
    k[high] = 0.0
    k[high, :, 0] = 25.0


@pytest.mark.parametrize("at", [(0, 5), (0, 70), (150, 5), (40, 190)], ids=str)
@pytest.mark.parametrize("heads", [(4, 2), (16, 16)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_seen_nan_of_weight_zero(dtype, d, heads, at):
    """(key with the high score, key with the NaN value) of one sequence between two others."""
    hq, hkv = heads
    lens, (high, nan) = [20, 200, 9], at
    q, k, v = (randn(i, sum(lens), h, d, dtype=TYPES[dtype][1]) for i, h in enumerate((hq, hkv, hkv)))
    far_apart(q, k, 20 + high)
    v[20 + nan, :, 3] = float("nan")
    a = make(dtype, hq, hkv, d, sum(lens), 3, scale=SCALE)
    out, lse = a.prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_of(lens))
    ref = R.prompt(q, k, v, lens, SCALE)
    assert torch.isnan(ref[0][20 + nan:220, :, 3]).all() and int(torch.isnan(ref[0]).sum()) == (200 - nan) * hq
    check(out, lse, ref, dtype)


@pytest.mark.parametrize("nan", [7, 100, 3000, 5000])
@pytest.mark.parametrize("n", [1, 6, 40])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cached_seen_nan_of_weight_zero(dtype, d, n, nan):
    """A tile cut into many parts: the high score lies in the first, the NaN in any of them."""
    hq, hkv, page = 4, 1, 32
    cache, keys, values = fill_cache(dtype, hkv, d, page, [5000 + n, 90 + n], seed=4)
    q = randn(1, 2 * n, hq, d, dtype=TYPES[dtype][1])
    far_apart(q, keys[0], 2)
    values[0][nan, :, 3] = float("nan")
    for pool, host in ((cache.k, keys[0]), (cache.v, values[0])):
        for slot in range(-(-host.shape[0] // page)):
            rows = host[slot * page:(slot + 1) * page]
            pool[1, int(cache.page_table[0, slot]), :, :rows.shape[0]] = rows.transpose(0, 1).to(DEV)
    a = make(dtype, hq, hkv, d, 2 * n, 2, scale=SCALE)
    out, lse = a.cached(q.to(DEV), cache, 1, ints([0, 1]), cu_of([n, n]))
    ref = R.cached(q, keys, values, [n, n], [seen_of(5000 + n, n, None), seen_of(90 + n, n, None)], SCALE)
    assert torch.isnan(ref[0][:n, :, 3]).all() and torch.isfinite(ref[0][n:]).all()
    check(out, lse, ref, dtype)
