"""Page operations of the cache against the host model: bookkeeping equal, data equal bit for bit."""
import numpy as np
import pytest
import torch

import serving_reference as R
from paper_2609_01024_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def ints(v):
    return torch.tensor(np.asarray(v, np.int32), device=DEV)


def cu_of(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]))


class Pair:
    """The library's cache and the model, driven side by side.  Pools hold distinct values, so a wrong row shows."""

    def __init__(self, pages=40, page=16, hkv=2, d=64, layers=3, max_seqs=12, max_pages=6, dtype=B.PCOMOE_BF16):
        self.c = B.PagedCache(layers=layers, pages=pages, page_size=page, kv_heads=hkv, head_dim=d, max_seqs=max_seqs,
                              max_pages=max_pages, dtype=dtype, device=DEV)
        g = torch.Generator().manual_seed(pages + page)
        dt = torch.bfloat16 if dtype == B.PCOMOE_BF16 else torch.float32
        self.k = torch.randn(layers, pages, hkv, page, d, generator=g).to(dt)
        self.v = torch.randn(layers, pages, hkv, page, d, generator=g).to(dt)
        self.c.k.copy_(self.k), self.c.v.copy_(self.v)
        self.b = R.Book(pages, page, max_seqs, max_pages)
        self.layers, self.hkv, self.d, self.dt, self.g = layers, hkv, d, dt, g

    def check(self, status=0):
        assert self.c.device_status() == status
        assert np.array_equal(self.c.seq_len.cpu().numpy(), self.b.len)
        assert np.array_equal(self.c.page_ref.cpu().numpy(), self.b.ref)
        assert np.array_equal(self.c.page_table.cpu().numpy(), self.b.table)
        assert torch.equal(self.c.k.cpu(), self.k) and torch.equal(self.c.v.cpu(), self.v)

    def move(self):
        for pool in (self.k, self.v):
            old = pool.clone()
            for a, b in self.b.moves:
                pool[:, b] = old[:, a]

    def reserve(self, seqs, add):
        self.c.reserve(ints(seqs), ints(add))
        self.b.reserve(seqs, add)
        self.move()

    def write(self, seqs, counts, layer=None):
        L = 1 if layer is not None else self.layers
        x = torch.randn(2, L, sum(counts), self.hkv, self.d, generator=self.g).to(self.dt)
        y = x.to(DEV)
        if layer is not None:
            self.c.write(y[0, 0], y[1, 0], ints(seqs), cu_of(counts), layer=layer)
        else:
            self.c.write(y[0], y[1], ints(seqs), cu_of(counts))
        t = 0
        for s, n in zip(seqs, counts):
            for j in range(n):
                p, r = self.b.place(s, int(self.b.len[s]) - n + j)
                for pool, src in ((self.k, x[0]), (self.v, x[1])):
                    lo = 0 if layer is None else layer
                    pool[lo:lo + L, p, :, r] = src[:, t]
                t += 1

    def fork(self, parents, children):
        self.c.fork(ints(parents), ints(children))
        self.b.fork(parents, children)

    def trim(self, seqs, lens):
        self.c.trim(ints(seqs), ints(lens))
        self.b.trim(seqs, lens)

    def keep(self, seqs, counts, keep):
        m = max(1, max(len(x) for x in keep))
        table = np.full((len(seqs), m), -1, np.int32)
        for i, x in enumerate(keep):
            table[i, :len(x)] = x
        self.c.keep(ints(seqs), cu_of(counts), ints(table), ints([len(x) for x in keep]))
        for s, n, x in zip(seqs, counts, keep):
            base = int(self.b.len[s]) - n
            for pool in (self.k, self.v):
                old = pool.clone()
                for j, m in enumerate(x):
                    (pa, ra), (pb, rb) = self.b.place(s, base + m), self.b.place(s, base + j)
                    pool[:, pb, :, rb] = old[:, pa, :, ra]
            self.b.trim([s], [base + len(x)])

    def compact(self):
        self.c.compact()
        self.b.compact()
        self.move()


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dtype", [B.PCOMOE_BF16, B.PCOMOE_FP32], ids=["bf16", "f32"])
def test_a_serving_turn(page, dtype):
    """Prompts, forks, growth with copies of shared pages, drafts kept and dropped, freeing, compaction."""
    p = Pair(page=page, dtype=dtype, d=128 if page == 32 else 64)
    p.reserve([0, 3, 1], [page + 5, 1, 2 * page]), p.check()
    p.write([0, 3, 1], [page + 5, 1, 2 * page]), p.check()
    p.fork([0, 0, 3], [5, 6, 7]), p.check()
    p.reserve([5, 0, 6, 1], [1, 1, 1, 1]), p.check()                # two copy the shared page, the last one keeps it
    p.write([5, 0, 6, 1], [1, 1, 1, 1], layer=1), p.check()
    p.reserve([7, 5, 3], [9, page + 3, 0]), p.check()
    p.write([7, 5], [9, page + 3]), p.check()
    p.keep([7, 5], [9, page + 3], [[0, 2, 3, 4, 5, 6, 7, 8], list(range(0, page + 3, 2))]), p.check()
    p.trim([0, 6], [0, 3]), p.check()
    p.compact(), p.check()
    p.compact(), p.check()                                            # nothing left to move
    p.reserve([0], [4 * page]), p.check()                             # the lowest free pages again


@pytest.mark.parametrize("seed", range(6))
def test_random_operations(seed):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([16, 32]))
    p = Pair(pages=int(rng.integers(30, 90)), page=page, max_seqs=9, max_pages=5, layers=2)
    for _ in range(40):
        what = rng.integers(6)
        seqs = [int(s) for s in rng.permutation(9)[:rng.integers(1, 9)]]
        if what <= 1:
            add = [int(rng.integers(0, min(2 * page, 5 * page - p.b.len[s]) + 1)) for s in seqs]
            worst = sum(p.b.need(a) + 2 for a in add)
            if worst <= int((p.b.ref == 0).sum()):
                p.reserve(seqs, add)
                p.write(seqs, add)
                if what == 1:
                    p.keep(seqs, add, [sorted(int(x) for x in rng.permutation(a)[:rng.integers(0, a + 1)]) for a in add])
        elif what == 2:
            empty, full = [s for s in seqs if p.b.len[s] == 0], [s for s in seqs if p.b.len[s] > 0]
            if empty and full:
                p.fork([full[int(rng.integers(len(full)))] for _ in empty], empty)
        elif what == 3:
            p.trim(seqs, [int(rng.integers(0, p.b.len[s] + 1)) for s in seqs])
        elif what == 4:
            p.trim(seqs[:2], [0] * len(seqs[:2]))
        else:
            p.compact()
        p.check()


def test_many_sequences_and_pages():
    """More sequences than threads of the planning block, and as many pages as several of its passes."""
    p = Pair(pages=6000, page=16, hkv=1, d=64, layers=1, max_seqs=1500, max_pages=4)
    seqs = list(np.random.default_rng(0).permutation(1500))
    p.reserve([int(s) for s in seqs], [int(17 + s % 20) for s in range(1500)]), p.check()
    p.trim([int(s) for s in seqs[::3]], [0] * 500), p.check()
    kids = [int(s) for s in seqs[::3]]
    p.fork([int(seqs[1])] * 500, kids), p.check()
    p.reserve(kids, [1] * 500), p.check()
    p.compact(), p.check()


def test_device_errors_leave_things_as_they_are():
    p = Pair(pages=8, max_pages=6)
    p.reserve([0, 1], [40, 20]), p.check()
    for seqs, add, status in (([2], [99], 7), ([2, 3], [60, 60], 8), ([2, 2], [1, 1], 7), ([12], [1], 7), ([-1], [1], 7), ([2], [-1], 7),
                              ([2, 3], [1, 97], 7)):
        p.c.reserve(ints(seqs), ints(add))
        p.check(status)
    for seqs, lens in (([0], [41]), ([0], [-1]), ([50], [0]), ([0, 0], [3, 5])):
        p.c.trim(ints(seqs), ints(lens))
        p.check(7)
    for parents, kids in (([0], [1]), ([0], [0]), ([0], [12]), ([-1], [3]), ([0, 1], [3, 3]), ([0, 3], [3, 4])):
        p.c.fork(ints(parents), ints(kids))
        if (parents, kids) == ([0, 3], [3, 4]):
            p.b.fork([3], [4])                                        # the other pair of that call is fine (an empty fork)
        p.check(7)
    x = torch.ones(8, 2, 64, dtype=torch.bfloat16, device=DEV)
    p.fork([0], [5]), p.check()
    p.c.write(x, x, ints([5]), ints([0, 8]), layer=0)                 # the last page is shared: not written
    p.check(7)
    p.c.write(x, x, ints([6]), ints([0, 8]), layer=0)                 # no such position
    p.check(7)
    for keep, n in (([[1, 1]], [2]), ([[2, 1]], [2]), ([[0, 8]], [2]), ([[1, 2]], [2]), ([[1, 2]], [3])):
        p.c.keep(ints([5]), ints([0, 8]), ints(keep), ints(n))        # not ascending, out of range, shared page, too many
        p.check(7)
    p.keep([1], [4], [[0, 3]]), p.check()


def test_refusals():
    import ctypes
    lib = B.load_library()
    p = Pair()
    ws, ok = p.c._ws, ints([0, 1])
    a = ok.data_ptr()
    size = ctypes.c_size_t(0)
    for field, value, status in (("page_size", 24, 4), ("page_size", 8, 4), ("head_dim", 4, 4), ("pages", 0, 1), ("dtype", 2, 1), ("max_seqs", 5000, 2),
                                 ("pages", (1 << 18) + 1, 2), ("d_k", None, 1), ("d_v", p.c.v.data_ptr() + 2, 4), ("struct_size", 1, 1), ("layers", -1, 1)):
        c = B.pcomoe_cache.from_buffer_copy(p.c.c)
        setattr(c, field, value)
        assert lib.pcomoe_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(size)) == status, field
        assert lib.pcomoe_cache_reserve(ctypes.byref(c), 1, a, a, *ws, None) == status, field
    assert lib.pcomoe_cache_workspace_bytes(p.c._ref, None) == 1
    assert lib.pcomoe_cache_reserve(p.c._ref, -1, a, a, *ws, None) == 1 and lib.pcomoe_cache_reserve(p.c._ref, 13, a, a, *ws, None) == 2
    assert lib.pcomoe_cache_reserve(p.c._ref, 1, None, a, *ws, None) == 1 and lib.pcomoe_cache_reserve(p.c._ref, 0, None, None, *ws, None) == 0
    assert lib.pcomoe_cache_reserve(p.c._ref, 1, a, a, ws[0], ws[1] - 1, None) == 3 and lib.pcomoe_cache_trim(p.c._ref, 1, a, a, None, 0, None) == 3
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    w = lambda layer=0, n_layers=1, T=2, rs=128, ls=0, k=x.data_ptr(): lib.pcomoe_cache_write(p.c._ref, layer, n_layers, T, 1, a, a, k, k, rs, ls, *ws, None)
    assert w(layer=3) == 1 and w(n_layers=4) == 1 and w(layer=-1) == 1 and w(T=-1) == 2 and w(rs=127) == 1 and w(k=None) == 1
    assert w(rs=132) == 4 and w(k=x.data_ptr() + 2) == 4 and w(T=0) == 0
    assert lib.pcomoe_cache_keep(p.c._ref, 1, a, a, None, 2, a, *ws, None) == 1
    assert lib.pcomoe_cache_fork(p.c._ref, 1, a, None, *ws, None) == 1
    p.check()
