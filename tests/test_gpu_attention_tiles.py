"""Prompts in the tensor-core kernel's larger form (256 rows to a tile, more pieces than SMs, rings that wrap inside a piece), called over
and over on one workspace; two objects at work at the same time.  Bounds as in test_gpu_attention."""
import pytest
import torch

import serving_reference as R
from test_gpu_attention import DEV, check, cu_of, fill_cache, ints, make, randn, seen_of

pytestmark = pytest.mark.gpu
SMS = 148


def tiles_of_256(hq, hkv, lens):
    """Whether the launch takes tiles of 256 rows."""
    return (sum(lens) * (hq // hkv) // 256 + len(lens)) * hkv >= SMS


def pieces(hq, hkv, lens):
    return sum(-(-n * (hq // hkv) // 256) for n in lens) * hkv


@pytest.mark.parametrize("hq,hkv,lens", [
    (32, 8, [1100, 700, 0, 1, 400]),                       # groups of 4: tokens of a tile 64, several tiles and 9 blocks of keys
    (32, 32, [1500]),                                      # one head to a group: 12 blocks of keys, the first half stops before the second
    (32, 16, [900, 129, 1]),
    (28, 4, [1490, 64, 31, 255]),                          # 7 does not divide a tile
    (48, 16, [770, 33])], ids=str)                         # nor does 3
@pytest.mark.parametrize("d", [64, 128])
def test_prompt_of_large_tiles(d, hq, hkv, lens):
    """Three heads of each against the definition; five calls on one workspace give the same bits everywhere."""
    assert tiles_of_256(hq, hkv, lens) and pieces(hq, hkv, lens) > SMS
    T, g = sum(lens), hq // hkv
    q, k, v = (randn(i + d, T, h, d, dtype=torch.bfloat16, std=1.2) for i, h in enumerate((hq, hkv, hkv)))
    x, cu = [y.to(DEV) for y in (q, k, v)], cu_of(lens)
    at = make("bf16", hq, hkv, d, T, len(lens))
    first = None
    for call in range(5):                                  # the counter of pieces is back at zero after each
        at.out.fill_(7.0)
        at.lse.fill_(7.0)
        out, lse = at.prompt(*x, cu)
        assert at.device_status() == 0
        if first is None:
            first = (out.clone(), lse.clone())
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), call
    for h in sorted({0, hq // 2 + 1, hq - 1}):
        one = lambda y, i: y[:, i:i + 1]
        check(one(out, h), one(lse, h), R.prompt(one(q, h), one(k, h // g), one(v, h // g), lens, d ** -0.5), "bf16")


def test_a_long_call_and_a_short_one_on_one_workspace():
    """Calls with more pieces than SMs and with fewer, packed and over a cache, in turn: each leaves the workspace as it found it."""
    hq, hkv, d, lens = 32, 8, 128, [1100, 700, 0, 1, 400]
    T = sum(lens)
    q, k, v = (randn(i, T, h, d, dtype=torch.bfloat16).to(DEV) for i, h in enumerate((hq, hkv, hkv)))
    cache, _, _ = fill_cache("bf16", hkv, d, 64, [3000, 200], seed=2)
    at = make("bf16", hq, hkv, d, T, 5)
    calls = [lambda: at.prompt(q, k, v, cu_of(lens)),
             lambda: at.prompt(q[:90], k[:90], v[:90], cu_of([40, 50])),
             lambda: at.cached(q[:2], cache, 1, ints([0, 1]), cu_of([1, 1])),
             lambda: at.cached(q[:80], cache, 1, ints([0, 1]), cu_of([40, 40]))]
    want = [[x.clone() for x in call()] for call in calls]
    for i in (0, 1, 0, 2, 0, 3, 1, 3, 2, 2, 0):
        out, lse = calls[i]()
        assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1]), i
    assert at.device_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_objects_at_the_same_time(dtype):
    """Prompts and cached calls of two objects with a workspace each, on two streams, do not touch one another."""
    hq, hkv, d, lens = 8, 2, 64, [700, 300]
    T = sum(lens)
    a, b = make(dtype, hq, hkv, d, T, 2), make(dtype, hq, hkv, d, T, 2)
    q, k, v = (randn(i, T, h, d, dtype=a.out.dtype).to(DEV) for i, h in enumerate((hq, hkv, hkv)))
    cache, keys, values = fill_cache(dtype, hkv, d, 32, [2000, 900], seed=3)
    cu, cu1, seqs = cu_of(lens), cu_of([20, 30]), ints([0, 1])
    want_p = [x.clone() for x in a.prompt(q, k, v, cu)]
    want_c = [x.clone() for x in b.cached(q[:50], cache, 1, seqs, cu1)]
    check(want_c[0], want_c[1], R.cached(q[:50].cpu(), keys, values, [20, 30], [seen_of(2000, 20, None), seen_of(900, 30, None)], d ** -0.5), dtype)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for i in range(20):
        for s, call in zip(streams, (lambda: a.prompt(q, k, v, cu), lambda: b.cached(q[:50], cache, 1, seqs, cu1))):
            with torch.cuda.stream(s):
                got.append([x.clone() for x in call()])
    torch.cuda.synchronize()
    for i in range(0, 40, 2):
        assert all(torch.equal(x, y) for x, y in zip(got[i], want_p)) and all(torch.equal(x, y) for x, y in zip(got[i + 1], want_c)), i
    assert a.device_status() == 0 and b.device_status() == 0
