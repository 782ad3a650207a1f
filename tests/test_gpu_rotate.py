"""Norm and rotation of heads against 64 bits: types, layouts, partial rotation, far positions, in place, into the cache."""
import numpy as np
import pytest
import torch

import turn_reference as ref
from paper_2609_01024_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (B.PCOMOE_BF16, torch.bfloat16), "f32": (B.PCOMOE_FP32, torch.float32)}
# Roundings of an element, in steps of 2^-24 of |a| + |b|: 19 of the sum of squares, half of them left by the root, 4 of rsqrt, 2 products,
# the angle (pi, from rounding the turn), 4 of sine and cosine, 3 of the products and their sum: below 32.  bf16 adds half a step of its own.
STEPS = 32 * 2.0 ** -24


def ints(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def close(got, want, dtype, size):
    got = got.double().cpu().numpy()
    bound = STEPS * size + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 0.0) * (1 + STEPS)
    if dtype == "bf16":
        bound = bound + STEPS * size * 2.0 ** -8
    assert (np.abs(got - want) <= bound + 1e-37).all(), float((np.abs(got - want) - bound).max())


def inputs(dtype, T, hq, hkv, d, rot, norm, seed=0, far=131072):
    t = TYPES[dtype][1]
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (torch.randn((T, (hq + 2 * hkv) * d), generator=g, device="cuda") * 1.7).to(t)
    q, k, v = qkv[:, :hq * d].unflatten(1, (hq, d)), qkv[:, hq * d:(hq + hkv) * d].unflatten(1, (hkv, d)), qkv[:, (hq + hkv) * d:].unflatten(1, (hkv, d))
    position = torch.randint(0, far, (T,), generator=g, device="cuda", dtype=torch.int32)
    inv_freq = torch.tensor(5e5 ** (-np.arange(rot // 2) / max(1, rot // 2)), dtype=torch.float64, device="cuda")
    w = [(torch.randn(d, generator=g, device="cuda") * 0.3 + 1).to(t) if norm else None for _ in range(2)]
    return q, k, v, position, inv_freq, w


def rotation(dtype, hq, hkv, d, inv_freq, neighbours, w, eps=1e-6):
    return B.HeadRotation(q_heads=hq, kv_heads=hkv, head_dim=d, inv_freq=inv_freq if len(inv_freq) else None, neighbours=neighbours, q_weight=w[0], k_weight=w[1], eps=eps,
                          dtype=TYPES[dtype][0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,neighbours", [(64, 64, False), (128, 128, False), (128, 128, True), (64, 64, True), (128, 48, False), (64, 16, True), (128, 112, False), (64, 0, False)])
@pytest.mark.parametrize("T,hq,hkv,norm", [(1, 8, 2, True), (3, 1, 1, True), (37, 28, 4, True), (300, 7, 7, False), (5, 5, 5, True)])
def test_packed(dtype, d, rot, neighbours, T, hq, hkv, norm):
    q, k, _, position, inv_freq, w = inputs(dtype, T, hq, hkv, d, rot, norm, seed=T + d + rot)
    f = rotation(dtype, hq, hkv, d, inv_freq, neighbours, w)
    qo, ko = torch.empty((T, hq, d), dtype=q.dtype, device="cuda"), torch.empty((T, hkv, d), dtype=q.dtype, device="cuda")
    kept = q.clone(), k.clone()
    f.rotate(q, k, position, qo, ko)
    assert torch.equal(q, kept[0]) and torch.equal(k, kept[1])
    for x, y, weight in ((q, qo, w[0]), (k, ko, w[1])):
        want, size = ref.rotate(x, weight, 1e-6, position.cpu().numpy(), inv_freq.cpu().numpy(), rot, neighbours)
        close(y, want, dtype, size)
    f.rotate(q, k, position)                   # over the inputs, column ranges of one projection
    assert torch.equal(q, qo) and torch.equal(k, ko)


@pytest.mark.parametrize("positions", [[0, 1, -1, -100000], [2 ** 31 - 1, -2 ** 31, 10 ** 9, 2 ** 24 + 1]])
def test_any_position(positions):
    q, k, _, _, inv_freq, w = inputs("f32", 4, 4, 2, 128, 128, True)
    f = rotation("f32", 4, 2, 128, inv_freq, False, w)
    position = ints(positions)
    qo, ko = torch.empty((4, 4, 128), device="cuda"), torch.empty((4, 2, 128), device="cuda")
    f.rotate(q, k, position, qo, ko)
    # 64-bit angles of positions up to 2^31: 2^31 * 2^-53 * 2 pi radians, far below fp32's steps, on both sides
    for x, y, weight in ((q, qo, w[0]), (k, ko, w[1])):
        want, size = ref.rotate(x, weight, 1e-6, positions, inv_freq.cpu().numpy(), 128, False)
        close(y, want, "f32", size * 1.25)


def test_one_weight_alone():
    """Queries normed, keys not."""
    q, k, _, position, inv_freq, w = inputs("bf16", 9, 8, 2, 128, 128, True)
    f = rotation("bf16", 8, 2, 128, inv_freq, False, (w[0], None))
    qo, ko = torch.empty((9, 8, 128), dtype=q.dtype, device="cuda"), torch.empty((9, 2, 128), dtype=q.dtype, device="cuda")
    f.rotate(q, k, position, qo, ko)
    for x, y, weight in ((q, qo, w[0]), (k, ko, None)):
        want, size = ref.rotate(x, weight, 1e-6, position.cpu().numpy(), inv_freq.cpu().numpy(), 128, False)
        close(y, want, "bf16", size)


def test_zero_rows_and_spoiled_heads():
    """A head of zeros stays zeros; a NaN or an infinity stays in its head."""
    q, k, _, position, inv_freq, w = inputs("bf16", 6, 8, 2, 128, 128, True)
    q, k = q.contiguous(), k.contiguous()
    f = rotation("bf16", 8, 2, 128, inv_freq, False, w)
    clean = [torch.empty_like(q), torch.empty_like(k)]
    f.rotate(q, k, position, *clean)
    q[1, 3] = 0
    q[2, 5, 17] = float("nan")
    k[4, 1, 0] = float("inf")
    out = [torch.empty_like(q), torch.empty_like(k)]
    f.rotate(q, k, position, *out)
    assert (out[0][1, 3] == 0).all() and torch.isnan(out[0][2, 5]).all() and torch.isnan(out[1][4, 1]).any()
    same = torch.ones((6, 8), dtype=torch.bool, device="cuda")
    same[1, 3] = same[2, 5] = False
    assert torch.equal(out[0][same], clean[0][same])
    same = torch.ones((6, 2), dtype=torch.bool, device="cuda")
    same[4, 1] = False
    assert torch.equal(out[1][same], clean[1][same])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hq,hkv,page", [(128, 8, 2, 16), (64, 3, 3, 64), (128, 32, 8, 128), (64, 5, 1, 32)])
@pytest.mark.parametrize("keys_out", [False, True])
def test_cached(dtype, d, hq, hkv, page, keys_out):
    """Rows of several sequences, an empty one among them, rows before and behind the list, two layers."""
    ctx, add = [0, 40, 7, 130, 15], [3, 1, 0, 70, 2]
    before, behind = 2, 3
    T = before + sum(add) + behind
    q, k, v, position, inv_freq, w = inputs(dtype, T, hq, hkv, d, d, True, seed=d)
    c = ref.cache_of(B, TYPES[dtype][0], layers=2, page=page, kv_heads=hkv, head_dim=d, lens=[x + y for x, y in zip(ctx, add)])
    f = rotation(dtype, hq, hkv, d, inv_freq, True, w)
    qo = torch.full((T, hq, d), 7.0, dtype=q.dtype, device="cuda")
    ko = torch.full((T, hkv, d), 7.0, dtype=q.dtype, device="cuda") if keys_out else None
    pools = c.k.clone(), c.v.clone()
    order = [3, 0, 2, 1, 4]                     # not that of their numbers
    cu = ints(before + np.concatenate([[0], np.cumsum([add[s] for s in order])]))
    f.rotate_cached(q, k, v, position, c, 1, ints(order), cu, qo, ko)
    torch.cuda.synchronize()
    assert c.device_status() == 0
    inside = slice(before, T - behind)
    for x, y, weight in ((q, qo, w[0]), (k, ko, w[1])):
        if y is None:
            continue
        want, size = ref.rotate(x[inside], weight, 1e-6, position[inside].cpu().numpy(), inv_freq.cpu().numpy(), d, True)
        close(y[inside], want, dtype, size)
        assert (y[:before] == 7).all() and (y[T - behind:] == 7).all()
    want_k, size = ref.rotate(k, w[1], 1e-6, position.cpu().numpy(), inv_freq.cpu().numpy(), d, True)
    at = before
    table = c.page_table.cpu().numpy()
    for s in order:
        for j in range(add[s]):
            p = ctx[s] + j
            place = (1, int(table[s, p // page]), slice(None), p % page)
            close(c.k[place], want_k[at], dtype, size[at])
            assert torch.equal(c.v[place], v[at])
            pools[0][place], pools[1][place] = c.k[place], c.v[place]
            at += 1
    assert torch.equal(c.k, pools[0]) and torch.equal(c.v, pools[1])          # nothing else was written


def test_refused_places():
    """A shared page, a sequence that is none, a list past T: reported, their keys are not cached, the others are."""
    q, k, v, position, inv_freq, w = inputs("bf16", 6, 8, 2, 64, 64, False)
    f = rotation("bf16", 8, 2, 64, inv_freq, False, w)
    c = ref.cache_of(B, B.PCOMOE_BF16, page=16, kv_heads=2, head_dim=64, lens=[20, 40])
    shared = int(c.page_table[1, 2])
    c.page_ref[shared] = 2
    kept = c.k.clone()
    qo = torch.empty((6, 8, 64), dtype=q.dtype, device="cuda")
    f.rotate_cached(q, k, v, position, c, 0, ints([0, 1]), ints([0, 2, 4]), qo)
    assert c.device_status() == 7 and c.device_status() == 0
    assert torch.equal(c.k[0, shared], kept[0, shared])
    page = int(c.page_table[0, 1])
    assert not torch.equal(c.k[0, page, :, 2:4], kept[0, page, :, 2:4])
    c.page_ref[shared] = 1
    for seqs, cu in (([0, -1], [0, 2, 4]), ([0, 9], [0, 2, 4]), ([0, 1], [0, 2, 8]), ([0, 1], [0, 2, 60])):
        f.rotate_cached(q, k, v, position, c, 0, ints(seqs), ints(cu), qo)
        assert c.device_status() == 7


def test_many_rows_and_graph():
    """A batch that takes several heads per warp gives the same bits as its rows alone, also from a graph on another stream."""
    T, hq, hkv, d = 4000, 32, 8, 128
    q, k, _, position, inv_freq, w = inputs("bf16", T, hq, hkv, d, d, True)
    f = rotation("bf16", hq, hkv, d, inv_freq, False, w)
    qo, ko = torch.empty((T, hq, d), dtype=q.dtype, device="cuda"), torch.empty((T, hkv, d), dtype=q.dtype, device="cuda")
    f.rotate(q, k, position, qo, ko)
    for lo, hi in ((0, 1), (1999, 2010), (3995, 4000)):
        a, b = torch.empty((hi - lo, hq, d), dtype=q.dtype, device="cuda"), torch.empty((hi - lo, hkv, d), dtype=q.dtype, device="cuda")
        f.rotate(q[lo:hi], k[lo:hi], position[lo:hi], a, b)
        assert torch.equal(a, qo[lo:hi]) and torch.equal(b, ko[lo:hi])
    want = qo.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            f.rotate(q, k, position, qo, ko)
        qo.zero_()
        graph.replay()
    side.synchronize()
    assert torch.equal(qo, want)
