"""Arguments of the serving calls that are refused before any device is touched."""
import ctypes

import pytest

from paper_2609_01024_b200 import binding


@pytest.fixture(scope="module")
def lib():
    from paper_2609_01024_b200 import build
    return binding.load_library(build.build())


def config(**kw):
    c = binding.pcomoe_attn_config(ctypes.sizeof(binding.pcomoe_attn_config), 8, 2, 128, binding.PCOMOE_BF16, 0.1)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


def cache(**kw):
    c = binding.pcomoe_cache(ctypes.sizeof(binding.pcomoe_cache), 2, 10, 16, 2, 128, binding.PCOMOE_BF16, 4, 5, 256, 512, 1024, 2048, 4096)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


@pytest.mark.parametrize("field,value,status", [("struct_size", 0, 1), ("q_heads", 7, 1), ("q_heads", 0, 1), ("kv_heads", -2, 1), ("head_dim", 80, 4),
                                                ("head_dim", 0, 1), ("dtype", 2, 1), ("scale", float("nan"), 1), ("scale", 0.0, 1), ("scale", -1.0, 1),
                                                ("q_heads", 8192, 2)])
def test_attention_config(lib, field, value, status):
    n = ctypes.c_size_t(0)
    assert lib.pcomoe_attn_workspace_bytes(config(**{field: value}), ctypes.byref(n)) == status
    assert lib.pcomoe_attn_prompt(config(**{field: value}), 0, 1, None, None, 0, None, 0, None, 0, None, 0, None, None, 0, None) == status


def test_attention_calls(lib):
    assert lib.pcomoe_attn_workspace_bytes(config(), None) == 1
    p = 4096
    f = lambda T=4, k=p, ks=256, v=p: lib.pcomoe_attn_prompt(config(), T, 1, p, p, 1024, k, ks, v, 256, p, 1024, None, None, 0, None)
    assert f(T=0) == 0 and f(T=-1) == 2 and f(k=None) == 1 and f(ks=255) == 1 and f(k=p + 8) == 4 and f(ks=260) == 4 and f(v=p + 2) == 4
    g = lambda c=cache(), layer=0, T=4, seqs=p, mask=None, words=0: lib.pcomoe_attn_cached(config(), c, layer, T, 1, seqs, p, p, 1024, mask, words, p, 1024, None,
                                                                                           None, 0, None)
    assert g(T=0) == 0 and g(T=-1) == 2 and g(layer=2) == 1 and g(layer=-1) == 1 and g(seqs=None) == 1 and g(mask=p) == 1 and g(words=9) == 2
    assert g(c=cache(head_dim=64)) == 1 and g(c=cache(kv_heads=4)) == 1 and g(c=cache(dtype=1)) == 1 and g(c=cache(page_size=48)) == 4 and g(c=None) == 1


@pytest.mark.parametrize("field,value,status", [("struct_size", 4, 1), ("layers", 0, 1), ("pages", -1, 1), ("pages", (1 << 18) + 1, 2), ("page_size", 256, 4),
                                                ("kv_heads", 0, 1), ("head_dim", 12, 4), ("dtype", 9, 1), ("max_seqs", 4097, 2), ("max_pages", 0, 1),
                                                ("max_pages", 1 << 28, 2), ("d_k", None, 1), ("d_seq_len", None, 1), ("d_v", 264, 4)])
def test_cache_layout(lib, field, value, status):
    n = ctypes.c_size_t(0)
    c = cache(**{field: value})
    assert lib.pcomoe_cache_workspace_bytes(c, ctypes.byref(n)) == status
    assert lib.pcomoe_cache_compact(c, None, 0, None) == status
    assert lib.pcomoe_cache_trim(c, 1, 256, 256, None, 0, None) == status


def test_cache_calls(lib):
    n = ctypes.c_size_t(0)
    assert lib.pcomoe_cache_workspace_bytes(cache(), ctypes.byref(n)) == 0 and n.value % 256 == 0 and n.value >= 256 + 3 * 40
    ws = (256, n.value, None)
    assert lib.pcomoe_cache_fork(cache(), -1, 256, 256, *ws) == 1 and lib.pcomoe_cache_fork(cache(), 5, 256, 256, *ws) == 2
    assert lib.pcomoe_cache_fork(cache(), 1, None, 256, *ws) == 1 and lib.pcomoe_cache_fork(cache(), 0, None, None, *ws) == 0
    assert lib.pcomoe_cache_fork(cache(), 1, 256, 256, 264, n.value, None) == 3 and lib.pcomoe_cache_fork(cache(), 1, 256, 256, 256, n.value - 1, None) == 3
    assert lib.pcomoe_cache_keep(cache(), 1, 256, 256, None, 3, 256, *ws) == 1 and lib.pcomoe_cache_keep(cache(), 1, 256, 256, 256, -1, 256, *ws) == 1


def test_scores(lib):
    f = lambda dtype=0, T=2, V=100, x=256, row=100, tok=256, top=0, lp=256, ids=None, best=None: lib.pcomoe_token_logprobs(dtype, T, V, x, row, tok, top, lp, None, ids,
                                                                                                                           best, None)
    assert f(T=0) == 0 and f(dtype=5) == 1 and f(T=-3) == 2 and f(V=0) == 2 and f(top=40) == 2 and f(V=2 << 20, row=2 << 20) == 4
    assert f(x=None) == 1 and f(x=257) == 1 and f(row=99) == 1 and f(tok=None) == 1 and f(lp=None) == 1 and f(top=2) == 1
