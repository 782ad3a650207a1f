"""Attention weight accumulated per cached position, against 64 bits; bounds count the kernel's fp32 steps."""
import numpy as np
import pytest
import torch

import turn_reference as ref
from paper_2609_01024_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (B.PCOMOE_BF16, torch.bfloat16), "f32": (B.PCOMOE_FP32, torch.float32)}


def ints(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


class Case:
    """A cache, packed queries, and the log sums that their attention would have left (fp32, rounded from 64 bits)."""

    def __init__(self, dtype, hq, hkv, d, page, ctx, add, kept=None, seed=0, order=None, behind=0, scale=None, layers=1, layer=0):
        self.__dict__.update(hq=hq, hkv=hkv, d=d, page=page, add=add, kept=kept, order=order or list(range(len(ctx))), layer=layer)
        code, t = TYPES[dtype]
        self.scale = d ** -0.5 if scale is None else scale
        rng = np.random.default_rng(seed)
        counted = [len(k) for k in kept] if kept else add
        self.lens = [c + m for c, m in zip(ctx, counted)]
        self.base = ctx
        self.cache = ref.cache_of(B, code, layers=layers, page=page, kv_heads=hkv, head_dim=d, lens=self.lens, room=[max(1, x) for x in self.lens], seed=seed)
        T = sum(add) + behind
        self.q = torch.tensor(rng.standard_normal((T, hq * d + 8)) * 2.0).to(t).cuda()[:, 8:].unflatten(1, (hq, d))     # rows of a wider array
        self.cu = np.concatenate([[0], np.cumsum([add[s] for s in self.order])])
        self.lse = torch.zeros((T, hq), device="cuda")
        self.weights = B.CacheWeights(self.cache, q_heads=hq, scale=scale)
        self.weights.weight.copy_(torch.tensor(rng.random(self.weights.weight.shape) * 2))
        self.rows = []                          # packed rows counted, in the list's order
        q = self.q.double().cpu().numpy()
        for i, s in enumerate(self.order):
            a = int(self.cu[i])
            mine = [a + x for x in (kept[s] if kept else range(add[s]))]
            self.rows.append(mine)
            k = self.keys(s)
            for n, row in enumerate(mine):
                for h in range(hq):
                    x = k[:self.base[s] + n + 1, h // (hq // hkv)] @ q[row, h] * self.scale
                    m = x.max()
                    self.lse[row, h] = float(m + np.log(np.exp(x - m).sum()))

    def keys(self, s):
        return ref.rows_of(self.cache.k[self.layer], self.cache.page_table[s].tolist(), self.page, self.lens[s]).double().cpu().numpy()

    def lists(self):
        if not self.kept:
            return {}
        width = max(1, max(len(k) for k in self.kept))
        return dict(keep=ints([list(self.kept[s]) + [-1] * (width - len(self.kept[s])) for s in self.order]), n_keep=ints([len(self.kept[s]) for s in self.order]))

    def add_up(self, fresh=True):
        self.weights.add(self.q, self.lse, self.layer, ints(self.order), ints(self.cu), fresh=fresh, **self.lists())

    def check(self, fresh=True):
        before = self.weights.weight.double().cpu().numpy()
        self.add_up(fresh)
        got = self.weights.weight.double().cpu().numpy()
        assert self.weights.device_status() == 0
        q, lse = self.q.double().cpu().numpy(), self.lse.double().cpu().numpy()
        for i, s in enumerate(self.order):
            n = self.lens[s] if self.rows[i] else 0
            assert np.array_equal(got[s, n:], before[s, n:])
            if not n:
                continue
            want, err = ref.weigh(q, lse, self.keys(s), self.scale, self.rows[i], self.base[s])
            old = before[s, :n].copy()
            if fresh:
                old[self.base[s]:] = 0
            bound = err + (np.abs(old) + want) * 2.0 ** -23
            assert (np.abs(got[s, :n] - old - want) <= bound).all(), float((np.abs(got[s, :n] - old - want) / bound).max())
            # the rows' weights add up to one a head and row
            if fresh:
                total = (got[s, :n] - old).sum()
                assert abs(total - len(self.rows[i]) * self.hq) <= bound.sum() + 2e-6 * total
        for s in range(len(self.lens)):
            if s not in self.order:
                assert np.array_equal(got[s], before[s])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 128, 16), (32, 8, 128, 64), (4, 4, 64, 16), (28, 4, 128, 32), (7, 1, 64, 128), (5, 5, 128, 64), (16, 1, 128, 16)])
def test_decode_step(dtype, hq, hkv, d, page):
    Case(dtype, hq, hkv, d, page, [300, 0, 1, 15, 16, 17, 129, 64], [1] * 8, seed=hq).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64), (12, 2, 64), (6, 3, 128)])
def test_kept_drafts(dtype, hq, hkv, d):
    """The kept rows of several drafts each, nothing kept, sequences in another order, rows behind the list."""
    kept = [[0, 2, 5], [], [0], [0, 1, 2, 3, 4, 6], [1]]
    c = Case(dtype, hq, hkv, d, 16, [100, 50, 0, 33, 700], [7, 3, 1, 7, 2], kept, seed=3, order=[4, 0, 3, 1], behind=3)
    c.check()
    c.check(fresh=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,ctx,add", [(8, 2, 128, [0], [130]), (4, 4, 64, [0, 77, 500], [65, 40, 33]), (2, 1, 128, [1000, 3], [9, 129]), (8, 8, 64, [0, 0, 0], [1, 64, 0]),
                                              (16, 2, 128, [200, 0], [40, 17]), (3, 1, 64, [20], [300])])
def test_prompts_and_chunks(dtype, hq, hkv, d, ctx, add):
    Case(dtype, hq, hkv, d, 32, ctx, add, seed=len(ctx)).check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_heads(dtype):
    """More kv heads than are held at a time, and groups of more heads than fit at once."""
    Case(dtype, 40, 40, 64, 16, [50, 33], [2, 1], seed=1).check()
    Case(dtype, 300, 1, 128, 16, [60], [2], seed=2).check()


def test_many_sequences():
    rng = np.random.default_rng(0)
    Case("bf16", 8, 2, 64, 16, rng.integers(0, 90, 150).tolist(), rng.integers(0, 3, 150).tolist(), seed=4, order=rng.permutation(150).tolist()).check()


def test_another_layer_and_scale():
    Case("bf16", 8, 2, 128, 16, [100, 5], [3, 1], seed=5, layers=3, layer=2, scale=0.02).check()


def test_two_layers_of_a_step():
    """The first layer sets the new positions, the others add to them."""
    c = Case("bf16", 8, 2, 64, 16, [40], [5], seed=6, layers=2)
    c.weights.weight[:, 40:45] = 1e30
    c.add_up(fresh=True)
    one = c.weights.weight.clone()
    assert float(one[0, 40:45].max()) < 100
    c.add_up(fresh=False)
    assert torch.allclose(c.weights.weight[0, 40:45], 2 * one[0, 40:45], rtol=2 ** -22)


def test_spoiled_keys_and_log_sums():
    """A NaN or infinite key spoils its own position alone; a position behind the row adds nothing; a row that saw nothing adds nothing."""
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 8, 2, 128, 16, [50], [4], seed=8)
        clean = c.weights.weight.clone()
        c.add_up()
        want, c.weights.weight[:] = c.weights.weight.clone(), clean
        page = lambda p: (0, int(c.cache.page_table[0, p // 16]), 0, p % 16)
        c.cache.k[page(7)] = float("nan")
        c.cache.k[page(53)] = float("nan")      # the last row's own
        c.cache.k[(0, int(c.cache.page_table[0, 3]), slice(None), slice(6, None))] = float("nan")      # behind the end
        c.add_up()
        got = c.weights.weight
        spoiled = torch.isnan(got[0])
        assert spoiled.nonzero().flatten().tolist() == [7, 53]
        keep = ~spoiled
        assert torch.equal(got[0][keep], want[0][keep])
        c.weights.weight[:] = clean
        c.cache.k[page(7)] = 0
        c.cache.k[page(53)] = 0
        c.lse[:] = float("-inf")
        c.add_up()
        assert torch.equal(c.weights.weight[0, :50], clean[0, :50]) and (c.weights.weight[0, 50:54] == 0).all()


def test_reported():
    c = Case("bf16", 8, 2, 64, 16, [30, 20, 10], [2, 2, 2], seed=9)
    before = c.weights.weight.clone()
    for order, cu in (([0, 0, 1], [0, 2, 4, 6]), ([0, 7, 1], [0, 2, 4, 6]), ([0, -1, 1], [0, 2, 4, 6]), ([0, 1, 2], [0, 2, 4, 90]), ([0, 1, 2], [0, 4, 2, 6])):
        c.weights.weight.copy_(before)
        c.weights.add(c.q, c.lse, 0, ints(order), ints(cu), fresh=True)
        assert c.weights.device_status() == 7 and c.weights.device_status() == 0
        if order == [0, 0, 1]:
            assert torch.equal(c.weights.weight[0], before[0]) and not torch.equal(c.weights.weight[1], before[1])
    # more rows than positions, numbers that are no rows
    c.weights.weight.copy_(before)
    c.cache.seq_len[2] = 1
    c.weights.add(c.q, c.lse, 0, ints([0, 1, 2]), ints([0, 2, 4, 6]))
    assert c.weights.device_status() == 7 and torch.equal(c.weights.weight[2], before[2]) and not torch.equal(c.weights.weight[1], before[1])
    c.weights.add(c.q, c.lse, 0, ints([0]), ints([0, 2]), keep=ints([[0, 5]]), n_keep=ints([2]))
    assert c.weights.device_status() == 7
    c.weights.add(c.q, c.lse, 0, ints([0]), ints([0, 2]), keep=ints([[0, 1]]), n_keep=ints([3]))
    assert c.weights.device_status() == 7


def test_bits_and_graph():
    """The same bits from call to call and from a graph; the graph replays with other lengths."""
    c = Case("bf16", 32, 8, 128, 16, [500, 90, 1300], [1, 4, 2], seed=10)
    before = c.weights.weight.clone()
    c.add_up()
    want = c.weights.weight.clone()
    args = (c.q, c.lse, 0, ints([0, 1, 2]), ints([0, 1, 5, 7]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.weights.add(*args, fresh=True)
        for _ in range(3):
            c.weights.weight.copy_(before)
            graph.replay()
            assert torch.equal(c.weights.weight, want)
        c.cache.seq_len[2] = 800
        c.weights.weight.copy_(before)
        graph.replay()
    side.synchronize()
    assert torch.equal(c.weights.weight[:2], want[:2]) and torch.equal(c.weights.weight[2, 800:], before[2, 800:])


def test_after_attention():
    """With the log sums of the attention call itself each row's weights add up to its heads: bf16 products twice, fp32 sums."""
    d, hq, hkv = 128, 16, 4
    c = Case("bf16", hq, hkv, d, 64, [900, 300], [3, 200], seed=12)
    attn = B.Attention(q_heads=hq, kv_heads=hkv, head_dim=d, max_tokens=203, max_seqs=2)
    _, lse = attn.cached(c.q, c.cache, 0, ints([0, 1]), ints([0, 3, 203]))
    c.weights.weight.zero_()
    c.weights.add(c.q, lse, 0, ints([0, 1]), ints([0, 3, 203]), fresh=True)
    total = c.weights.weight.double().sum(1).cpu().numpy()
    # every term of a row has the same relative error of its log sum (|lse| up to 60: 60 * 2^-23) and its own of its score
    assert np.allclose(total, [3 * hq, 200 * hq], rtol=2e-5)


@pytest.mark.parametrize("hq,hkv,d,page,ctx,add", [(32, 8, 128, 64, [0], [700]), (8, 8, 64, 16, [130, 0, 1000], [257, 128, 90]), (28, 4, 128, 32, [5], [300]), (6, 2, 128, 128, [0, 0, 0, 60], [200, 0, 1, 333]),
                                                   (4, 1, 64, 16, [2000], [150]), (10, 10, 128, 16, [77], [129]), (7, 1, 128, 64, [0], [1000]), (32, 8, 128, 16, [500], [30]),
                                                   (8, 2, 64, 32, [9] * 40, [24] * 39 + [100])])
def test_many_rows(hq, hkv, d, page, ctx, add):
    """Column tiles that groups of heads do not divide, units without columns, more steps than there are places for log sums, fewer rows
    than a tile holds, more sequences than a warp has lanes."""
    c = Case("bf16", hq, hkv, d, page, ctx, add, seed=hq + d, behind=5)
    c.check()
    c.check(fresh=False)


def test_many_kept_rows():
    """Lists of many rows, some numbers left out, beside sequences with none."""
    rng = np.random.default_rng(1)
    kept = [sorted(rng.permutation(400)[:300].tolist()), [], [0, 2], list(range(150))]
    Case("bf16", 8, 2, 128, 32, [40, 30, 0, 500], [400, 3, 3, 150], kept, seed=2, order=[3, 2, 1, 0]).check()


def test_many_rows_spoiled():
    """In the tensor-core kernel too a key spoils its own position alone and rows that saw nothing, or are no rows, add nothing."""
    c = Case("bf16", 8, 2, 128, 16, [50], [300], seed=13)
    clean = c.weights.weight.clone()
    c.add_up()
    want, c.weights.weight[:] = c.weights.weight.clone(), clean
    page = lambda p: (0, int(c.cache.page_table[0, p // 16]), 0, p % 16)
    c.cache.k[page(7)] = float("nan")
    c.cache.k[page(349)] = float("nan")
    c.cache.k[page(200)] = float("inf")
    c.add_up()
    got = c.weights.weight
    spoiled = torch.isnan(got[0]) | torch.isinf(got[0]) | (got[0] != want[0])
    assert spoiled.nonzero().flatten().tolist() == [7, 200, 349]
    c.weights.weight[:] = clean
    for p in (7, 200, 349):
        c.cache.k[page(p)] = 1.0
    c.q[10] = float("nan")                      # a row that saw nothing, whatever it holds
    c.lse[10] = float("-inf")
    c.add_up()
    assert torch.isfinite(c.weights.weight).all()
    rows = torch.arange(300, device="cuda") != 10
    keep = ints([[i if i != 10 else 1000 for i in range(300)]])
    c.weights.weight[:] = clean
    c.weights.add(c.q, c.lse, 0, ints([0]), ints([0, 300]), keep=keep, n_keep=ints([300]), fresh=True)
    assert c.weights.device_status() == 7 and torch.isfinite(c.weights.weight).all()


def test_many_rows_bits_and_graph():
    c = Case("bf16", 16, 4, 128, 64, [300, 0], [200, 400], seed=14)
    before = c.weights.weight.clone()
    c.add_up()
    want = c.weights.weight.clone()
    args = (c.q, c.lse, 0, ints([0, 1]), ints([0, 200, 600]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.weights.add(*args, fresh=True)
        for _ in range(5):
            c.weights.weight.copy_(before)
            graph.replay()
            assert torch.equal(c.weights.weight, want)
    side.synchronize()
    assert c.weights.device_status() == 0


def test_two_objects_at_once():
    """Both kernels, on two streams at the same time, give the bits that they give alone."""
    cases = [Case("bf16", 16, 4, 128, 64, [300, 0], [200, 400], seed=15), Case("bf16", 32, 8, 128, 16, [500, 90, 1300], [1, 4, 2], seed=16), Case("bf16", 8, 8, 64, 16, [70], [500], seed=17),
             Case("f32", 8, 2, 64, 16, [400, 33], [3, 1], seed=18)]
    before = [c.weights.weight.clone() for c in cases]
    want, args = [], []
    for c in cases:
        c.add_up()
        want.append(c.weights.weight.clone())
        args.append((ints(c.order), ints(c.cu)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):
        for st, c, b, a in zip(streams, cases, before, args):
            with torch.cuda.stream(st):
                c.weights.weight.copy_(b)
                c.weights.add(c.q, c.lse, 0, *a, fresh=True)
    torch.cuda.synchronize()
    assert all(torch.equal(c.weights.weight, w) and c.weights.device_status() == 0 for c, w in zip(cases, want))


def test_weights_in_a_wider_array_and_few_listed():
    c = Case("bf16", 8, 2, 128, 16, [100, 60, 40], [2, 120, 1], seed=19, order=[1, 2])
    before = c.weights.weight.clone()
    c.add_up()
    want = c.weights.weight.clone()
    room = c.weights.weight.shape[1]
    wide = torch.full((before.shape[0], room + 40), 3.0, device="cuda")
    w = B.CacheWeights(c.cache, q_heads=8, weight=wide[:, 8:8 + room], max_listed=2)
    w.weight.copy_(before)
    w.add(c.q, c.lse, 0, ints(c.order), ints(c.cu), fresh=True)
    assert torch.equal(w.weight, want) and (wide[:, :8] == 3).all() and (wide[:, 8 + room:] == 3).all() and w.device_status() == 0


@pytest.mark.parametrize("hq,hkv,d,page,ctx,add", [(32, 8, 128, 64, [0], [150]), (8, 8, 64, 16, [130, 0, 300], [57, 128, 33]), (28, 4, 128, 32, [5], [80]), (6, 2, 128, 128, [0, 0, 0, 60], [200, 0, 1, 133]),
                                                   (4, 1, 64, 16, [700], [65]), (7, 1, 128, 64, [0], [300]), (3, 3, 64, 32, [9] * 40, [50] * 39 + [64])])
def test_many_rows_f32(hq, hkv, d, page, ctx, add):
    """Tiles of 64 columns and keys that end everywhere, sequences without rows, more sequences than a warp has lanes."""
    c = Case("f32", hq, hkv, d, page, ctx, add, seed=hq + d, behind=5)
    c.check()
    c.check(fresh=False)


def test_many_kept_rows_f32():
    rng = np.random.default_rng(1)
    kept = [sorted(rng.permutation(200)[:150].tolist()), [], [0, 2], list(range(90))]
    Case("f32", 8, 2, 128, 32, [40, 30, 0, 100], [200, 3, 3, 90], kept, seed=2, order=[3, 2, 1, 0]).check()


def test_many_rows_spoiled_f32():
    c = Case("f32", 8, 2, 128, 16, [50], [300], seed=13)
    clean = c.weights.weight.clone()
    c.add_up()
    want, c.weights.weight[:] = c.weights.weight.clone(), clean
    page = lambda p: (0, int(c.cache.page_table[0, p // 16]), 0, p % 16)
    for p, x in ((7, float("nan")), (349, float("nan")), (200, float("inf"))):
        c.cache.k[page(p)] = x
    c.cache.k[(0, int(c.cache.page_table[0, 21]), slice(None), slice(14, None))] = float("nan")      # behind the end
    c.q[10] = float("nan")                      # a row that saw nothing, whatever it holds
    c.lse[10] = float("-inf")
    c.add_up()
    first, c.weights.weight[:] = c.weights.weight.clone(), clean
    c.add_up()
    assert torch.equal(torch.nan_to_num(first, nan=-1.0, posinf=-2.0), torch.nan_to_num(c.weights.weight, nan=-1.0, posinf=-2.0))
    bad = ~torch.isfinite(first[0])
    assert bad[[7, 349]].all() and bad.nonzero().flatten().tolist() in ([7, 349], [7, 200, 349])
    keep = ~bad & (torch.arange(first.shape[1], device="cuda") != 200)
    # a row less: no more than before at every other position
    assert (first[0][keep] <= want[0][keep]).all()


@pytest.mark.parametrize("hq,hkv,d,ctx,add", [(6, 2, 64, [3000, 10, 2500, 700] * 2, [40, 1, 42, 60] * 2), (3, 1, 128, [4000, 3999], [50, 43]), (7, 1, 64, [6000], [20]),
                                              (6, 2, 64, [1500] * 19, [106, 3, 212] * 6 + [90]), (12, 4, 128, [2000] * 3, [33, 90, 1])])
def test_units_without_columns(hq, hkv, d, ctx, add):
    """Few tiles of columns and several shares of them: many units have nothing to do, and the copies of the units around them are still
    handed on (groups of heads that do not divide a tile)."""
    c = Case("bf16", hq, hkv, d, 32, ctx, add, seed=len(ctx) + hq)
    c.check()
    kept = [list(range(0, a, 1 + i % 2)) for i, a in enumerate(add)]
    Case("bf16", hq, hkv, d, 32, ctx, add, kept, seed=hq).check()


@pytest.mark.parametrize("dtype,hq,hkv,drafts,kept", [("bf16", 8, 2, 48, 3), ("bf16", 32, 8, 24, 6), ("f32", 8, 2, 9, 2), ("f32", 16, 4, 40, 7), ("bf16", 8, 2, 48, 30), ("f32", 8, 2, 9, 9)])
def test_kept_rows_of_many_drafts(dtype, hq, hkv, drafts, kept):
    """The kernel is chosen by the rows that may count, not by the rows that were drafted: one launch where lists of a few rows name them, two (partial
    sums and their join) from 96 columns a sequence on, in fp32 32."""
    rng = np.random.default_rng(drafts)
    lists = [sorted(rng.permutation(drafts)[:int(rng.integers(0, kept + 1))].tolist()) for _ in range(5)] + [list(range(kept))]
    c = Case(dtype, hq, hkv, 128, 16, [200, 0, 33, 500, 64, 17], [drafts] * 6, lists, seed=kept)
    c.check()
    before = B.pcomoe_launch_count()
    c.add_up()
    assert B.pcomoe_launch_count() - before == (2 if kept * (hq // hkv) >= (96 if dtype == "bf16" else 32) else 1)
