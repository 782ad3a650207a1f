"""NaN and infinities in values: what a row sees counts however small its weight, what it does not see never does.

One key scores 100 above the others, so that the others' weights (e^-100 = 2^-144) are zero in fp32 and not in the 64-bit
definition: a NaN among their values has to come out, wherever a block of keys is masked or a tile is cut.  The bounds are those of
test_gpu_attention; lse is then a number of size 100 behind five roundings of 2^-24 (scale times log2 e, the product with the
score, ln 2, the product with it, the sum): 100 * 5 * 2^-24 = 3e-5, inside the 1e-4 that `check` allows."""
import numpy as np
import pytest
import torch

import serving_reference as R
from paper_2609_01024_b200 import binding as B
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


def check_values(out, lse, ref, dtype):
    """`check`, and infinities are the reference's own."""
    inf = torch.isinf(ref[0])
    assert torch.equal(out.double().cpu()[inf], ref[0][inf])
    check(out, lse, ref, dtype)


def spoil(v, kind, T):
    """Values of one kv head and column, or of all of them, made NaN or infinite; returns v."""
    nan, inf = float("nan"), float("inf")
    if kind == "first":
        v[0, :, 3] = inf
    elif kind == "middle":
        v[T // 2, 0, 5], v[min(T // 2 + 1, T - 1), -1, 0] = nan, -inf
    elif kind == "last":
        v[T - 1] = nan
    elif kind == "everywhere":                                        # a value in every block of keys, in other columns
        for i, p in enumerate(range(5, T, 61)):
            v[p, i % v.shape[1], (7 * i) % v.shape[2]] = nan if i % 3 else inf
    elif kind == "all":
        v[:] = nan
    return v


KINDS = ["first", "middle", "last", "everywhere", "all"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,lens", [((2, 2), [300, 64]), ((7, 1), [210]), ((32, 8), [1100, 90])], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompt_values(dtype, d, heads, lens, kind):
    """Every row against the definition, in tiles of 128 and 256 rows; of 32 heads three."""
    hq, hkv = heads
    T, g = sum(lens), hq // hkv
    q, k, v = (randn(i, T, h, d, dtype=TYPES[dtype][1]) for i, h in enumerate((hq, hkv, hkv)))
    spoil(v, kind, lens[0])
    a = make(dtype, hq, hkv, d, T, len(lens))
    out, lse = a.prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_of(lens))
    assert a.device_status() == 0
    for h in sorted({0, hq // 2, hq - 1}):
        one = lambda x, i: x[:, i:i + 1]
        check_values(one(out, h), one(lse, h), R.prompt(one(q, h), one(k, h // g), one(v, h // g), lens, d ** -0.5), dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 7, 40, 90])
@pytest.mark.parametrize("tree", [False, True], ids=["chain", "tree"])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 128)])
def test_cached_values(dtype, d, tree, n, kind):
    """The same among drafted tokens and their contexts, whole and cut tiles."""
    hq, hkv, page, full = 4, 2, 32, [700 + n, 0 + n]
    cache, keys, values = fill_cache(dtype, hkv, d, page, full, seed=4)
    for s, m in enumerate(full):
        new = values[s][-n:]
        spoil(values[s] if kind == "first" else new, kind, n)
        for slot in range(-(-m // page)):
            rows = values[s][slot * page:(slot + 1) * page]
            cache.v[1, int(cache.page_table[s, slot]), :, :rows.shape[0]] = rows.transpose(0, 1).to(DEV)
    q = randn(1, 2 * n, hq, d, dtype=TYPES[dtype][1])
    trees = [R.tree_bits(np.random.default_rng(s), n) if tree else None for s in range(2)]
    a = make(dtype, hq, hkv, d, 2 * n, 2)
    out, lse = a.cached(q.to(DEV), cache, 1, ints([0, 1]), cu_of([n, n]), R.pack_bits(trees, 3).to(DEV) if tree else None)
    assert a.device_status() == 0
    check_values(out, lse, R.cached(q, keys, values, [n, n], [seen_of(m, n, t) for m, t in zip(full, trees)], d ** -0.5), dtype)


@pytest.mark.parametrize("at", [0, 2900, 4095])
def test_rows_formed_again_run_into_no_wait_limit(at):
    """A prompt of 4096 tokens with an infinity in one value, under a wait limit of 1 ms (a tile takes some 20 us): forming rows again
    is not a wait that ran out, and where every row sees the value (at 0) none is formed again."""
    T, h, d = 4096, 16, 128
    q, k, v = (randn(i, T, h, d, dtype=torch.bfloat16).to(DEV) for i in range(3))
    clean, cu = v.clone(), cu_of([T])
    v[at, :, 3] = float("inf")
    a = make("bf16", h, h, d, T, 1)
    want = a.prompt(q, k, clean, cu)[0].clone()

    def time(values):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        a.prompt(q, k, values, cu)
        end.record()
        end.synchronize()
        return begin.elapsed_time(end)
    plain = min(time(clean) for _ in range(5))
    try:
        B.pcomoe_set_wait_limit_us(1000)
        again = min(time(v) for _ in range(3))
        assert a.device_status() == 0
    finally:
        B.pcomoe_set_wait_limit_us(0)
    assert torch.isposinf(a.out[at:, :, 3]).all()
    keep = [c for c in range(d) if c != 3]
    assert torch.equal(a.out[:at], want[:at]) or float((a.out[:at].float() - want[:at].float()).abs().max()) <= 2 * 2.0 ** -8 * float(want.float().abs().max())
    assert torch.isfinite(a.out[:at]).all() and torch.isfinite(a.out[:, :, keep]).all()
    if at == 0:
        assert torch.equal(a.out[:, :, keep], want[:, :, keep])
        assert again < 20 * plain, (again, plain)
