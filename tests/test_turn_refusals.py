"""Arguments of the rotation, verification, weighing and eviction calls that are refused before any device is touched."""
import ctypes

import pytest

from paper_2609_01024_b200 import binding


@pytest.fixture(scope="module")
def lib():
    from paper_2609_01024_b200 import build
    return binding.load_library(build.build())


def made(cls, values, changes):
    c = cls(ctypes.sizeof(cls), *values)
    for k, v in changes.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def rotation(**kw):
    return made(binding.pcomoe_rotate_config, (8, 2, 128, 128, 0, binding.PCOMOE_BF16, 1e-6), kw)


def heads(**kw):
    return made(binding.pcomoe_attn_config, (8, 2, 128, binding.PCOMOE_BF16, 0.1), kw)


def cache(**kw):
    return made(binding.pcomoe_cache, (2, 10, 16, 2, 128, binding.PCOMOE_BF16, 4, 5, 256, 512, 1024, 2048, 4096), kw)


@pytest.mark.parametrize("field,value,status", [("struct_size", 0, 1), ("q_heads", 0, 1), ("kv_heads", -1, 1), ("head_dim", 0, 1), ("head_dim", 192, 4), ("rot_dim", -16, 1),
                                                ("rot_dim", 144, 1), ("rot_dim", 40, 4), ("pairs", 2, 1), ("dtype", 3, 1), ("eps", -1.0, 1), ("eps", float("nan"), 1),
                                                ("eps", float("inf"), 1), ("q_heads", 5000, 2), ("kv_heads", 5000, 2)])
def test_rotation_config(lib, field, value, status):
    assert lib.pcomoe_heads_rotate(rotation(**{field: value}), 0, *[None] * 4, *[None, 0] * 4, None) == status
    assert lib.pcomoe_heads_rotate_cached(rotation(**{field: value}), cache(), 0, 0, 0, *[None] * 6, *[None, 0] * 5, 256, 256, None) == status


def test_rotation_calls(lib):
    p = 4096

    def f(T=4, position=p, freq=p, qw=None, q=p, qs=1024, k=p, ks=256, qo=p, qos=1024, ko=p, kos=256, **kw):
        return lib.pcomoe_heads_rotate(rotation(**kw), T, position, freq, qw, None, q, qs, k, ks, qo, qos, ko, kos, None)
    assert f(T=0) == 0 and f(T=-1) == 2
    for missing in ("position", "freq", "q", "k", "qo", "ko"):
        assert f(**{missing: None}) == 1
    for short in ("qs", "ks", "qos", "kos"):
        assert f(**{short: 255}) == 1
    assert f(q=p + 8) == 4 and f(k=p + 2) == 4 and f(qo=p + 4) == 4 and f(ko=p + 8) == 4 and f(qw=p + 8) == 4 and f(freq=p + 4) == 4
    assert f(qs=1028) == 4 and f(ks=260) == 4 and f(qos=1025) == 4 and f(kos=257) == 4

    def g(T=4, n=2, c=cache(), layer=0, seqs=p, cu=p, v=p, vs=256, ko=None, ws=256, size=256, **kw):
        return lib.pcomoe_heads_rotate_cached(rotation(**kw), c, layer, T, n, seqs, cu, p, p, None, None, p, 1024, p, 256, v, vs, p, 1024, ko, 0, ws, size, None)
    assert g(T=0) == 0 and g(n=0) == 0 and g(T=-1) == 2 and g(n=-1) == 1 and g(n=5) == 2 and g(layer=2) == 1 and g(layer=-1) == 1
    assert g(seqs=None) == 1 and g(cu=None) == 1 and g(v=None) == 1 and g(vs=255) == 1 and g(v=p + 8) == 4 and g(vs=260) == 4 and g(ko=p) == 1
    assert g(c=None) == 1 and g(c=cache(head_dim=64)) == 1 and g(c=cache(kv_heads=4)) == 1 and g(c=cache(dtype=1)) == 1 and g(c=cache(page_size=48)) == 4
    assert g(ws=None) == 3 and g(ws=264) == 3 and g(size=255) == 3


def test_weigh(lib):
    n = ctypes.c_size_t(0)
    assert lib.pcomoe_weigh_workspace_bytes(heads(), cache(), 4, ctypes.byref(n)) == 0 and n.value >= 256
    assert lib.pcomoe_weigh_workspace_bytes(heads(), cache(), 4, None) == 1 and lib.pcomoe_weigh_workspace_bytes(heads(), cache(), -1, ctypes.byref(n)) == 1
    assert lib.pcomoe_weigh_workspace_bytes(heads(), cache(), 5, ctypes.byref(n)) == 2 and lib.pcomoe_weigh_workspace_bytes(None, cache(), 1, ctypes.byref(n)) == 1
    for bad, status in ((dict(head_dim=96), 4), (dict(q_heads=7), 1), (dict(scale=0.0), 1), (dict(dtype=5), 1), (dict(q_heads=8192), 2), (dict(kv_heads=4), 1)):
        assert lib.pcomoe_weigh_workspace_bytes(heads(**bad), cache(), 1, ctypes.byref(n)) == status
    lib.pcomoe_weigh_workspace_bytes(heads(), cache(), 2, ctypes.byref(n))
    size, p = n.value, 4096

    def f(layer=0, T=4, k=2, seqs=p, cu=p, q=p, qs=1024, lse=p, keep=None, ks=0, n_keep=None, w=p, wstride=80, ws=256, size=size):
        return lib.pcomoe_cache_weigh(heads(), cache(), layer, T, k, seqs, cu, q, qs, lse, keep, ks, n_keep, 0, w, wstride, ws, size, None)
    assert f(T=0) == 0 and f(k=0) == 0 and f(T=-1) == 2 and f(k=-1) == 1 and f(k=5) == 2 and f(layer=2) == 1
    for missing in ("seqs", "cu", "q", "lse", "w"):
        assert f(**{missing: None}) == 1
    assert f(keep=p, ks=3) == 1 and f(n_keep=p) == 1 and f(keep=p, ks=0, n_keep=p) == 1 and f(qs=1023) == 1 and f(wstride=79) == 1
    assert f(q=p + 8) == 4 and f(qs=1028) == 4 and f(ws=None) == 3 and f(ws=264) == 3 and f(size=size - 1) == 3


def test_evict(lib):
    n = ctypes.c_size_t(0)
    assert lib.pcomoe_evict_workspace_bytes(cache(), 3, ctypes.byref(n)) == 0 and n.value >= 256 + 3 * 8 * 80
    assert lib.pcomoe_evict_workspace_bytes(cache(), 5, ctypes.byref(n)) == 2 and lib.pcomoe_evict_workspace_bytes(cache(), -1, ctypes.byref(n)) == 1
    assert lib.pcomoe_evict_workspace_bytes(cache(), 1, None) == 1 and lib.pcomoe_evict_workspace_bytes(None, 1, ctypes.byref(n)) == 1
    lib.pcomoe_evict_workspace_bytes(cache(), 2, ctypes.byref(n))
    size, p = n.value, 4096

    def f(k=2, seqs=p, budget=p, sinks=0, recent=0, w=p, wstride=80, ws=256, size=size, **kw):
        return lib.pcomoe_cache_evict(cache(**kw), k, seqs, budget, sinks, recent, w, wstride, ws, size, None)
    assert f(k=0) == 0 and f(k=-1) == 1 and f(k=5) == 2 and f(sinks=-1) == 1 and f(recent=-1) == 1 and f(seqs=None) == 1 and f(budget=None) == 1 and f(w=None) == 1
    assert f(wstride=79) == 1 and f(ws=None) == 3 and f(ws=300) == 3 and f(size=size - 1) == 3 and f(page_size=20) == 4 and f(d_k=None) == 1 and f(layers=40000) == 2


def test_verify(lib):
    n = ctypes.c_size_t(0)
    assert lib.pcomoe_verify_workspace_bytes(10, ctypes.byref(n)) == 0 and n.value >= 256 + 160
    assert lib.pcomoe_verify_workspace_bytes(10, None) == 1 and lib.pcomoe_verify_workspace_bytes(-1, ctypes.byref(n)) == 2
    size, p = n.value, 4096

    def f(dtype=0, T=10, V=100, k=2, cu=p, tokens=p, x=p, stride=100, near=None, ns=0, u=p, un=p, keep=p, ks=4, nk=p, nxt=p, ws=256, size=size):
        return lib.pcomoe_verify_drafts(dtype, T, V, k, cu, tokens, None, x, stride, near, ns, None, u, un, keep, ks, nk, nxt, ws, size, None)
    assert f(k=0) == 0 and f(dtype=7) == 1 and f(T=-1) == 2 and f(V=0) == 2 and f(k=-1) == 2 and f(k=70000) == 2 and f(ks=-1) == 2 and f(V=(1 << 20) + 1, stride=1 << 21) == 4
    for missing in ("cu", "tokens", "x", "u", "un", "keep", "nk", "nxt"):
        assert f(**{missing: None}) == 1
    assert f(ks=0) == 1 and f(stride=99) == 1 and f(x=p + 1) == 1 and f(near=p, ns=99) == 1 and f(near=p + 2, ns=100) == 1
    assert f(ws=None) == 3 and f(ws=257) == 3 and f(size=size - 1) == 3


def test_verify_outputs_among_inputs(lib):
    """Each array at a place of its own; then an output at or inside of an input."""
    names = ("cu", "x", "near", "temperature", "u_next", "tokens", "parent", "u", "keep", "n_keep", "nxt")
    place = {k: 4096 * (i + 1) for i, k in enumerate(names)}

    def f(**at):
        a = dict(place, **at)
        return lib.pcomoe_verify_drafts(1, 10, 100, 2, a["cu"], a["tokens"], a["parent"], a["x"], 100, a["near"], 100, a["temperature"], a["u"], a["u_next"], a["keep"], 4,
                                        a["n_keep"], a["nxt"], 1 << 20, 4096, None)
    for out in ("keep", "n_keep", "nxt"):
        for i in ("cu", "temperature", "u_next", "x", "near"):
            assert f(**{out: place[i]}) == 1 and f(**{out: place[i] + 4}) == 1, (out, i)
        assert f(**{out: place["x"] + 3996}) == 1 and f(**{out: place["near"] + 3996}) == 1
