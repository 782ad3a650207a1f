"""Eviction by weight: which positions stay, their rows and weights in order, the pages given back."""
import numpy as np
import pytest
import torch

import turn_reference as ref
from paper_2609_01024_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": B.PCOMOE_BF16, "f32": B.PCOMOE_FP32}


def ints(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def make(dtype, lens, page=16, layers=2, hkv=2, d=64, seed=0):
    c = ref.cache_of(B, TYPES[dtype], layers=layers, page=page, kv_heads=hkv, head_dim=d, lens=lens, room=[max(1, x) for x in lens], seed=seed)
    w = B.CacheWeights(c, q_heads=hkv)
    rng = np.random.default_rng(seed)
    x = np.exp(rng.standard_normal(w.weight.shape) * 2).astype(np.float32)
    x[rng.random(x.shape) < 0.2] = 0.0
    w.weight.copy_(torch.tensor(x))
    return c, w


def check(c, w, seqs, budget, sinks, recent, untouched=()):
    lens, table = c.seq_len.tolist(), c.page_table.cpu().numpy().copy()
    weight, refs = w.weight.cpu().numpy().copy(), c.page_ref.cpu().numpy().copy()
    k, v = c.k.clone(), c.v.clone()
    w.evict(ints(seqs), ints(budget), sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    for s, n in enumerate(lens):
        b = budget[seqs.index(s)] if s in seqs and s not in untouched else n
        stays = ref.evict(weight[s], n, b, sinks, recent)
        assert int(c.seq_len[s]) == len(stays)
        used, had = -(-len(stays) // c.page_size), -(-n // c.page_size)
        assert c.page_table[s].tolist() == [int(table[s, j]) if j < used or j >= had else -1 for j in range(table.shape[1])]
        for j in range(used, had):
            refs[table[s, j]] -= 1
        assert np.array_equal(w.weight[s, :len(stays)].cpu().numpy(), weight[s, stays], equal_nan=True)
        assert np.array_equal(w.weight[s, len(stays):].cpu().numpy(), weight[s, len(stays):], equal_nan=True)
        for y in (k, v):
            for j, p in enumerate(stays):
                if j != p:
                    y[:, int(table[s, j // c.page_size]), :, j % c.page_size] = y[:, int(table[s, p // c.page_size]), :, p % c.page_size].clone()
    assert np.array_equal(c.page_ref.cpu().numpy(), refs)
    assert torch.equal(c.k, k) and torch.equal(c.v, v)


@pytest.mark.parametrize("dtype,d,page,layers,hkv", [("bf16", 64, 16, 2, 2), ("bf16", 128, 64, 1, 8), ("f32", 64, 32, 3, 1), ("f32", 128, 16, 1, 3), ("bf16", 72, 16, 1, 2)])
def test_layouts(dtype, d, page, layers, hkv):
    lens = [300, 0, 1, 17, 90, 1100, 64]
    c, w = make(dtype, lens, page, layers, hkv, d, seed=d)
    check(c, w, [5, 0, 3, 6, 1, 2], [700, 40, 16, 64, 0, 1], 2, 8)
    assert w.device_status() == 0
    check(c, w, [0, 5], [10, 10], 2, 8)         # again, from what the first one left
    assert w.device_status() == 0


@pytest.mark.parametrize("sinks,recent,budget", [(0, 0, 0), (0, 0, 1), (4, 0, 4), (0, 16, 16), (4, 16, 20), (4, 16, 21), (0, 0, 199), (0, 199, 199), (199, 0, 199), (0, 0, 200), (50, 50, 500)])
def test_budgets(sinks, recent, budget):
    c, w = make("bf16", [200, 33], seed=3)
    check(c, w, [0], [budget], sinks, recent)
    assert w.device_status() == 0


def test_ties_and_strange_weights():
    """Equal weights keep the lower positions; -0 is 0; infinities and negative ones have their place, a NaN is the lightest."""
    c, w = make("bf16", [500, 500, 500], seed=4)
    w.weight[0] = 1.0
    w.weight[1] = torch.tensor([0.0, -0.0, 1.0, -1.0, float("inf"), float("-inf"), float("nan"), 1e-42], device="cuda").repeat(64)[:w.weight.shape[1]]
    w.weight[2] = float("nan")
    for b in (400, 313, 250, 190, 100, 63, 7):
        check(c, w, [0, 1, 2], [b, b, b], 1, 3)
    assert w.device_status() == 0


def test_long_sequences():
    """Windows of the move and runs of the warps that end everywhere."""
    for n, b in ((20000, 15001), (33000, 513), (4097, 4096), (9000, 8191)):
        c, w = make("bf16", [n, 700], page=128, layers=1, hkv=1, seed=n)
        w.weight[0, : n // 2] += 1.0             # what stays lies in both halves
        check(c, w, [0, 1], [b, 699], 4, 64)


def test_many_pages():
    """More pages are given back than one block has threads, by sequences of very different lengths."""
    c, w = make("bf16", [30000, 10, 9000, 16400], page=16, layers=1, hkv=1, seed=21)
    check(c, w, [2, 0, 3, 1], [40, 20, 16399, 0], 4, 8, untouched=(1,))
    assert w.device_status() == 7               # a budget of 0 leaves no room for 4 + 8
    held = [t[t >= 0].tolist() for t in c.page_table]
    assert sorted(sum(held, [])) == c.page_ref.nonzero().flatten().tolist()


def test_weights_in_a_wider_array_and_few_listed():
    """Rows of weights that the caller has, further apart than they are long, and a workspace for two sequences at a time."""
    c, w0 = make("bf16", [300, 200, 100, 50], seed=22)
    wide = torch.full((w0.weight.shape[0], w0.weight.shape[1] + 96), 7.0, device="cuda")
    w = B.CacheWeights(c, q_heads=2, weight=wide[:, 32:32 + w0.weight.shape[1]], max_listed=2)
    w.weight.copy_(w0.weight)
    check(c, w, [3, 0], [20, 133], 2, 9)
    check(c, w, [2, 1], [99, 17], 2, 9)
    assert w.device_status() == 0 and (wide[:, :32] == 7).all() and (wide[:, -64:] == 7).all()
    with pytest.raises(AssertionError):
        w.evict(ints([0, 1, 2]), ints([5, 5, 5]))


def test_two_objects_at_once():
    """Two caches are cut down on two streams at the same time, again and again."""
    pairs = [make("bf16", [5000, 3000, 0, 700], page=16, layers=2, seed=s) for s in (23, 24)]
    want = []
    for c, w in pairs:
        state = [c.k.clone(), c.v.clone(), w.weight.clone(), c.seq_len.clone(), c.page_ref.clone(), c.page_table.clone()]
        w.evict(ints([1, 0, 3]), ints([900, 901, 902]), sinks=3, recent=50)
        want.append((state, [x.clone() for x in (c.k, c.v, w.weight, c.seq_len, c.page_ref, c.page_table)]))
    seqs, budget = ints([1, 0, 3]), ints([900, 901, 902])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(5):
        for st, (c, w), (state, _) in zip(streams, pairs, want):
            with torch.cuda.stream(st):
                for x, y in zip((c.k, c.v, w.weight, c.seq_len, c.page_ref, c.page_table), state):
                    x.copy_(y)
                w.evict(seqs, budget, sinks=3, recent=50)
    torch.cuda.synchronize()
    for (c, w), (_, after) in zip(pairs, want):
        assert all(torch.equal(x, y) for x, y in zip((c.k, c.v, w.weight, c.seq_len, c.page_ref, c.page_table), after)) and w.device_status() == 0


def test_shared_pages():
    """A fork's pages: a sequence that would write into them stays as it is and is reported; one that only gives them back is cut."""
    c, w = make("bf16", [100, 0, 60], seed=6)
    c.fork(ints([0]), ints([1]))
    check(c, w, [0, 2], [50, 20], 0, 0, untouched=(0,))
    assert w.device_status() == 7
    w.weight[1, :64] = 5.0                       # the first 64 stay: no row moves
    w.weight[1, 64:] = 1.0
    n_before = int(c.page_ref[int(c.page_table[1, 5])])
    page = int(c.page_table[1, 5])
    w.evict(ints([1]), ints([64]))
    assert w.device_status() == 0 and int(c.seq_len[1]) == 64 and int(c.page_ref[page]) == n_before - 1 and int(c.seq_len[0]) == 100


def test_reported():
    c, w = make("bf16", [100, 80, 60], seed=7)
    check(c, w, [0, 1], [-1, 70], 0, 0, untouched=(0,))
    assert w.device_status() == 7
    check(c, w, [0, 2], [10, 50], 8, 8, untouched=(0,))
    assert w.device_status() == 7
    lens = c.seq_len.tolist()
    for seqs in ([0, 0], [5, -1], [9, 9]):
        w.evict(ints(seqs), ints([20] * len(seqs)))
        assert w.device_status() == 7 and c.seq_len.tolist() == lens
    c.page_table[2, 1] = 10 ** 6                # no page
    w.evict(ints([2]), ints([20]))
    assert w.device_status() == 7 and c.seq_len.tolist() == lens


def test_graph():
    c, w = make("bf16", [400, 300], seed=8)
    seqs, budget = ints([0, 1]), ints([390, 290])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lens = []
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            w.evict(seqs, budget, sinks=1, recent=5)
        for b in (390, 200, 200, 33):
            budget.fill_(b)
            before, order = w.weight.cpu().numpy(), c.seq_len.tolist()
            graph.replay()
            lens.append(c.seq_len.tolist())
            for s in range(2):
                stays = ref.evict(before[s], order[s], b, 1, 5)
                assert np.array_equal(w.weight[s, :len(stays)].cpu().numpy(), before[s, stays])
    assert lens == [[390, 300], [200, 200], [200, 200], [33, 33]] and w.device_status() == 0
