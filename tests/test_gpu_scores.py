"""Token scores against the 64-bit definition.

Bounds: logZ is an fp32 number m + ln s whose rounding is 2^-24 |logZ|, s has relative error below 1e-5 (sums of at most 2^20
positive terms in 256 lanes and more, each exponential good to 2^-21), so a log probability is within
1e-5 + 2^-22 (|x| + |logZ|) and the entropy (terms p ln p, sum of them at most ln V) within 3e-5.  Ids are equal."""
import numpy as np
import pytest
import torch

import serving_reference as R
from paper_2609_01024_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def check(x, tokens, top, view=None):
    """x on the CPU; view: the device tensor to pass in its place."""
    y = x.to(DEV) if view is None else view
    s = B.TokenScores(max_tokens=x.shape[0], top_n=top, device=DEV)
    lp, ent, ids, best = (t.cpu() for t in s.score(y, torch.tensor(tokens, dtype=torch.int32, device=DEV)))
    want = R.scores(x, tokens, top)
    size = torch.where(torch.isfinite(x), x.double().abs(), torch.zeros((), dtype=torch.float64)).amax(1)     # of each row
    bound = 1e-5 + 2.0 ** -22 * 2 * size
    for got, ref, b in ((lp, want[0], bound), (ent, want[1], torch.full_like(bound, 3e-5)), (best, want[3], bound[:, None].expand(want[3].shape))):
        f = torch.isfinite(ref)
        assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[torch.isinf(ref)].double(), ref[torch.isinf(ref)])
        assert ((got.double() - ref)[f].abs() <= b[f]).all(), float((got.double() - ref)[f].abs().max())
    assert torch.equal(ids, want[2]), (ids, want[2])


def logits(seed, T, V, dtype, std=3.0):
    return (torch.randn(T, V, generator=torch.Generator().manual_seed(seed)) * std).to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 31, 127, 128, 129, 255, 256, 257, 1000, 4095, 5003, 50257])
@pytest.mark.parametrize("top", [0, 1, 5, 32])
def test_sizes(V, top, dtype):
    x = logits(V, 3, V, dtype)
    check(x, [0, V - 1, V // 2], top)


@pytest.mark.parametrize("T", [1, 40, 300, 700])
def test_rows(T):
    """Few rows are cut over a cluster of blocks, many are not."""
    x = logits(T, T, 9001, "bf16")
    check(x, [(7 * t) % 9001 for t in range(T)], 6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0, 1, 3, 5])
def test_strides_and_alignment(dtype, offset):
    T, V = 5, 3001
    whole = torch.full((T, V + 9), float("nan"), dtype=TYPES[dtype])
    whole[:, offset:offset + V] = logits(offset, T, V, dtype)
    d = whole.to(DEV)
    check(whole[:, offset:offset + V], [5, 0, V - 1, 17, 2999], 8, view=d[:, offset:offset + V])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 20000])
def test_ties_and_orders(dtype, V):
    rows = torch.stack([torch.zeros(V),                                              # all equal
                        torch.arange(V).float() / V,                                  # ascending (many bf16 ties)
                        -torch.arange(V).float() / V,
                        (torch.arange(V) % 3).float(),
                        torch.where(torch.arange(V) % 997 == 5, torch.tensor(4.0), torch.tensor(-4.0)),
                        torch.full((V,), -0.0) + torch.where(torch.arange(V) % 2 == 1, 0.0, -0.0)]).to(TYPES[dtype])
    if V == 20000:
        rows = rows[:5]
    check(rows + 0.0, [0, 1, V - 1, 7, 5, 9][:rows.shape[0]], 32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_and_extreme(dtype):
    V = 2500
    low = torch.finfo(TYPES[dtype]).min
    x = logits(1, 9, V, dtype)
    x[0] = float("-inf")                                                             # nothing eligible
    x[1, :] = float("-inf")
    x[1, 77] = 3.0                                                                   # one word
    x[2] = float("nan")
    x[2, 5], x[2, 6] = 1.0, float("inf")
    x[3] = low                                                                       # the lowest value is a value
    x[4, ::2] = low
    x[5, 100:] = float("-inf")
    x[6, 3], x[6, 9] = float("inf"), float("nan")
    x[7] = x[7] * 0 + torch.finfo(TYPES[dtype]).max
    x[8, :] = 1e4
    x[8, 0] = 1.0e4 + 64
    check(x, [3, 77, 6, 2, 0, 200, 3, 1, 0], 12)


def test_tokens_that_are_none():
    x = logits(3, 4, 100, "f32")
    check(x, [-1, 100, 2 ** 31 - 1, -7], 3)


def test_without_tokens_or_entropy():
    x = logits(3, 4, 1000, "f32").to(DEV)
    ids, lp = torch.zeros(4, 2, dtype=torch.int32, device=DEV), torch.zeros(4, 2, device=DEV)
    assert B.load_library().pcomoe_token_logprobs(B.PCOMOE_FP32, 4, 1000, x.data_ptr(), 1000, None, 2, None, None, ids.data_ptr(), lp.data_ptr(), None) == 0
    want = R.scores(x.cpu(), [0] * 4, 2)
    torch.cuda.synchronize()
    assert torch.equal(ids.cpu(), want[2])


def test_refusals():
    lib = B.load_library()
    x = torch.zeros(4, 64, device=DEV)
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    f = lambda dtype=1, T=4, V=64, x=x.data_ptr(), stride=64, tok=t.data_ptr(), top=0, lp=x.data_ptr(), ids=None, best=None: lib.pcomoe_token_logprobs(
        dtype, T, V, x, stride, tok, top, lp, None, ids, best, None)
    assert f(T=0) == 0 and f(dtype=2) == 1 and f(T=-1) == 2 and f(V=0) == 2 and f(top=33) == 2 and f(top=-1) == 2
    assert f(V=(1 << 20) + 1, stride=1 << 21) == 4 and f(x=None) == 1 and f(stride=63) == 1 and f(top=3) == 1 and f(lp=None) == 1 and f(tok=None) == 1
    assert f(x=x.data_ptr() + 2) == 1
