"""Objects of one GPU used while another one is current, on the host: the library launches on the current device, so that has to be
the object's own during a call, and the caller's again afterwards.  CUDA is stood in for by a record of what was current."""
import contextlib
import ctypes

import pytest
import torch

from paper_2609_01024_b200 import binding as B

OWN, OTHER = torch.device("cuda", 1), torch.device("cuda", 0)


class Stand:
    """What the binding looks at of a device tensor."""

    def __init__(self, *shape, dtype=torch.int32, device=OWN, at=4096):
        self.shape, self.dtype, self.device, self.at = shape, dtype, device, at

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def stride(self, i=None):
        s = [1]
        for x in reversed(self.shape[1:]):
            s.insert(0, s[0] * x)
        return tuple(s) if i is None else s[i]

    def get_device(self):
        return self.device.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at

    def __getitem__(self, _):
        return self


@pytest.fixture
def gpus(monkeypatch):
    """Device 0 is current.  Returns the record of (call, device current while it was made, stream handle)."""
    now, calls = [0], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], torch.device(d).index if not isinstance(d, int) else d
        try:
            yield
        finally:
            now[0] = before

    class Library:
        def __getattr__(self, name):
            def call(*args):
                calls.append((name, now[0], args[-1]))
                if name.endswith("workspace_bytes"):
                    ctypes.cast(args[-1], ctypes.POINTER(ctypes.c_size_t))[0] = 1024
                return 0
            call.__name__ = name
            return call

    def set_device(_):
        raise AssertionError("the caller's device is the caller's")

    library = Library()
    monkeypatch.setattr(B, "load_library", lambda path=None: library)
    monkeypatch.setattr(B, "_raw_stream", lambda i: 100 + i)
    monkeypatch.setattr(B, "_stream", lambda: 100 + now[0])
    monkeypatch.setattr(B, "_current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "set_device", set_device)
    for name in ("empty", "zeros"):
        real = getattr(torch, name)
        monkeypatch.setattr(torch, name, lambda *a, real=real, device=None, **kw: real(*a, **kw))
    return calls, now


def cache_on(device):
    c = object.__new__(B.PagedCache)
    c.device, c.gpu, c.kv_heads, c.head_dim, c.page_size, c.dtype = device, device.index, 2, 64, 16, B.PCOMOE_BF16
    c.c = B.pcomoe_cache()
    c._ref, c._ws, c.workspace, c._lib = ctypes.byref(c.c), (4096, 1024), Stand(1024), B.load_library()
    return c


def attention():
    return B.Attention(q_heads=4, kv_heads=2, head_dim=64, max_tokens=8, max_seqs=2, device="cuda:1")


def rows(heads, device=OWN):
    return Stand(3, heads, 64, dtype=torch.bfloat16, device=device)


def lse(device=OWN):
    return Stand(3, 4, dtype=torch.float32, device=device)


USES = {
    "reserve": lambda: cache_on(OWN).reserve(Stand(2), Stand(2)),
    "write": lambda: cache_on(OWN).write(rows(2), rows(2), Stand(2), Stand(3)),
    "fork": lambda: cache_on(OWN).fork(Stand(2), Stand(2)),
    "keep": lambda: cache_on(OWN).keep(Stand(2), Stand(3), Stand(2, 5), Stand(2)),
    "trim": lambda: cache_on(OWN).trim(Stand(2), Stand(2)),
    "compact": lambda: cache_on(OWN).compact(),
    "cache status": lambda: cache_on(OWN).device_status(),
    "prompt": lambda: attention().prompt(rows(4), rows(2), rows(2), Stand(3), out=rows(4), lse=lse()),
    "cached": lambda: attention().cached(rows(4), cache_on(OWN), 0, Stand(2), Stand(3), out=rows(4), lse=lse()),
    "attention status": lambda: attention().device_status(),
    "scores": lambda: B.TokenScores(max_tokens=8, top_n=2, device="cuda:1").score(Stand(3, 50, dtype=torch.float32), Stand(3)),
}


@pytest.mark.parametrize("use", USES)
@pytest.mark.parametrize("current", [0, 1])
def test_calls_run_on_the_objects_device(gpus, use, current):
    calls, now = gpus
    now[0] = current
    USES[use]()
    name, device, stream = calls[-1]
    assert device == 1 and stream == 101, calls
    assert now[0] == current
    assert all(d == 1 for _, d, _ in calls)                          # the constructors' questions too (the SM count is a device's)


def test_a_device_without_a_number_is_the_current_one(gpus):
    _, now = gpus
    now[0] = 1
    assert B.TokenScores(max_tokens=1, device="cuda").device == OWN


def test_a_refusal_names_the_call(gpus):
    a = attention()

    def refuse(*_):
        return 4
    refuse.__name__ = "pcomoe_attn_prompt"
    a._lib = type("L", (), {"pcomoe_attn_prompt": staticmethod(refuse)})
    with pytest.raises(B.PcomoeError, match="pcomoe_attn_prompt: PCOMOE_ERR_UNSUPPORTED"):
        a.prompt(rows(4), rows(2), rows(2), Stand(3), out=rows(4), lse=lse())
    assert gpus[1][0] == 0


@pytest.mark.parametrize("what", ["q", "cache", "out", "lse", "seqs"])
def test_tensors_of_another_device_are_refused(gpus, what):
    calls, _ = gpus
    a = attention()
    del calls[:]
    at = lambda name: OTHER if name == what else OWN
    with pytest.raises(AssertionError):
        a.cached(rows(4, at("q")), cache_on(at("cache")), 0, Stand(2, device=at("seqs")), Stand(3), out=rows(4, at("out")), lse=lse(at("lse")))
    assert not calls
