"""Verification of drafts: the walk and the next token equal those of 64 bits, at every size and kind of draft."""
import numpy as np
import pytest
import torch

import turn_reference as ref
from paper_2609_01024_b200 import binding as B

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def floats(v):
    return torch.tensor(np.asarray(v, np.float32), device="cuda")


def case(seed, V, add, tree, drafts, dtype, spread=2.0):
    rng = np.random.default_rng(seed)
    T = sum(add)
    x = rng.standard_normal((T, V)) * spread
    hot = rng.integers(0, V, (T, 4))
    np.put_along_axis(x, hot, np.take_along_axis(x, hot, 1) + 5.0, 1)
    x[rng.random((T, V)) < 0.05] = -np.inf
    y = np.where(np.isfinite(x), x, -3.0) + rng.standard_normal((T, V)) * 0.8
    near = np.exp(y - y.max(1, keepdims=True))
    near = (near / near.sum(1, keepdims=True)).astype(np.float32)
    parent, tokens = [], []
    at = 0
    for n in add:
        up = ([-1] + [int(rng.integers(0, j)) if tree else j - 1 for j in range(1, n)])[:n]
        for j in range(n):
            row = near[at + max(0, up[j])].astype(np.float64)
            tokens.append(int(rng.choice(V, p=row / row.sum())) if drafts else int(np.argsort(-row)[min(V - 1, rng.integers(0, 3))]))
        parent += up
        at += n
    return dict(x=torch.tensor(x).to(TYPES[dtype]).cuda(), tokens=tokens, cu=np.concatenate([[0], np.cumsum(add)]), parent=parent if tree else None,
                near=near if drafts else None, u=rng.random(T).astype(np.float32), u_next=rng.random(len(add)).astype(np.float32))


def run(c, temperature=None, most=None, x=None, near=None, verifier=None):
    add = np.diff(c["cu"])
    most = most or int(max(1, add.max()))
    v = verifier or B.DraftVerifier(max_seqs=len(add), max_path=most, max_tokens=max(1, int(add.sum())))
    near = near if near is not None else None if c["near"] is None else torch.tensor(c["near"], device="cuda")
    keep, n_keep, nxt = v.verify(c["x"] if x is None else x, ints(c["tokens"]), ints(c["cu"]), floats(c["u"]), floats(c["u_next"]),
                                 parent=None if c["parent"] is None else ints(c["parent"]), draft_probs=near,
                                 temperature=None if temperature is None else floats(temperature))
    keep, n_keep, nxt = keep.tolist(), n_keep.tolist(), nxt.tolist()
    return [k[:m] for k, m in zip(keep, n_keep)], nxt, keep, v


def same(c, temperature=None, most=None, **kw):
    got, nxt, keep, v = run(c, temperature, most, **kw)
    want = ref.verify(c["x"].double().cpu().numpy(), c["tokens"], c["cu"], c["u"], c["u_next"], c["parent"], c["near"], temperature, most or int(max(1, np.diff(c["cu"]).max())))
    assert got == want[0] and nxt == want[1], (got, want[0], nxt, want[1])
    for row, path in zip(keep, got):
        assert all(k == -1 for k in row[len(path):])
    return got, nxt, v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 33, 255, 256, 1000, 4097, 32000])
@pytest.mark.parametrize("tree,drafts", [(False, True), (False, False), (True, True), (True, False)])
def test_against_64_bits(dtype, V, tree, drafts):
    add = [5, 1, 9, 0, 3, 12]
    for seed in range(3):
        _, _, v = same(case(100 * seed + V, V, add, tree, drafts, dtype), [0.7, 1.0, 0.0, 1.0, 1.5, 0.3])
        assert v.device_status() == 0


@pytest.mark.parametrize("dtype,V,n", [("bf16", 151936, 2), ("f32", 151936, 1), ("f32", 1 << 20, 1), ("bf16", 128256, 40), ("bf16", 300, 300), ("f32", 50000, 160)])
def test_large(dtype, V, n):
    """Every split of rows over blocks and clusters."""
    for tree, drafts in ((False, True), (True, False)):
        same(case(V + n, V, [3] * n if V * n > 10 ** 7 else [4] * n, tree, drafts, dtype))


def test_next_token_at_every_border():
    """u_next at 0, just below 1 and between; many words of nearly the same probability."""
    rng = np.random.default_rng(0)
    n, V = 64, 5000
    c = case(1, V, [1] * n, False, False, "f32", spread=0.01)
    c["u_next"] = np.concatenate([[0.0, np.float32(1 - 2.0 ** -24), 0.5, 0.25], rng.random(n - 4)]).astype(np.float32)
    _, nxt, _ = same(c)
    assert len(set(nxt)) > n // 2


def test_tests_at_their_border():
    """u on either side of p / q by one step of fp32: 64 bits decide."""
    V, n = 1000, 64
    c = case(7, V, [2] * n, False, True, "f32")
    x = c["x"].double().cpu().numpy()
    for i in range(n):
        a = 2 * i
        p, q = ref.target(x[a], 1.0)[c["tokens"][a + 1]], float(c["near"][a, c["tokens"][a + 1]])
        edge = np.float32(min(p / q, 1 - 2.0 ** -24))
        c["u"][a + 1] = edge if i % 3 == 0 else np.nextafter(edge, np.float32(0)) if i % 3 == 1 else np.nextafter(edge, np.float32(1))
    same(c)


def test_given_drafts_named_twice():
    """Siblings with the same token: the second one's is gone; all of the mass refused: the target's own again."""
    V = 6
    x = np.log(np.array([[0.5, 0.3, 0.1, 0.05, 0.03, 0.02]] * 6))
    c = dict(x=torch.tensor(x, dtype=torch.float32).cuda(), tokens=[0, 0, 0, 1, 0, 2], cu=np.array([0, 6]), parent=[-1, 0, 0, 0, 0, 0], near=None,
             u=np.array([0, .9, .0, .99, .0, .999], np.float32), u_next=np.array([.1], np.float32))
    got, nxt, _ = same(c)
    assert got == [[0]] and nxt[0] in (3, 4, 5)
    one = np.full((3, V), -np.inf)
    one[:, 4] = 1.0                             # all of p on one word, which is refused by u = 1
    c = dict(x=torch.tensor(one, dtype=torch.float32).cuda(), tokens=[0, 4, 4], cu=np.array([0, 3]), parent=[-1, 0, 0], near=None, u=np.array([0, 1, 1], np.float32),
             u_next=np.array([.7], np.float32))
    got, nxt, _, _ = run(c)
    assert got == [[0]] and nxt == [4]


def test_not_finite_logits_and_probabilities():
    V, add = 700, [4, 4, 1, 3]
    c = case(3, V, add, False, True, "bf16")
    c["x"][0, ::3] = float("nan")
    c["x"][1, 5] = float("inf")
    c["x"][4] = float("-inf")                   # the second sequence's first row: nothing eligible
    c["x"][8] = float("nan")                    # and the third's
    c["near"][9, :50] = np.nan
    c["near"][9, 50:60] = -1
    c["near"][10, 3] = np.inf
    c["x"][9:12] += 0
    got, nxt, _ = same(c)
    assert got[1] == [0] and nxt[1] == -1 and nxt[2] == -1
    same(dict(c, near=None), [0.0, 0.0, 0.0, 0.5])


@pytest.mark.parametrize("temperature", [1e-30, 1e-4, 50.0, 1e30, 0.0, -1.0, float("inf"), float("nan")])
def test_temperatures(temperature):
    c = case(11, 999, [4, 6, 2], True, True, "f32")
    same(c, [temperature] * 3)
    c["x"] = c["x"] * 1e4                       # logits far apart
    same(c, [temperature] * 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_words_ruled_out_at_large_temperatures(dtype):
    """At a temperature of 1e30 the eligible words are all but equally likely, and -inf still has no weight; the type's largest logits apart."""
    rng = np.random.default_rng(2)
    n, V = 200, 4
    x = np.tile(np.array([0.0, -np.inf, 1.0, -np.inf]), (2 * n, 1))
    c = dict(x=torch.tensor(x).to(TYPES[dtype]).cuda(), tokens=rng.choice([0, 2], 2 * n).tolist(), cu=np.arange(n + 1) * 2, parent=None, near=None,
             u=rng.random(2 * n).astype(np.float32), u_next=rng.random(n).astype(np.float32))
    got, _, _ = same(c, [1e30] * n)
    assert 0.3 * n < sum(len(g) > 1 for g in got) < 0.7 * n
    big = float(torch.finfo(TYPES[dtype]).max)
    c["x"] = torch.tensor(np.tile(np.array([-big, -np.inf, big, 0.0]), (2 * n, 1))).to(TYPES[dtype]).cuda()
    got, nxt, _ = same(c, [1e38] * n)
    assert len(set(nxt)) == 3 or min(len(g) for g in got) == 1
    same(c, [1.0] * n)


def test_greedy_takes_the_lowest_of_the_best():
    x = torch.zeros((3, 4000), device="cuda")
    x[:, [17, 900, 3999]] = 2.0
    x[0, 5] = -0.0
    c = dict(x=x, tokens=[1, 900, 17], cu=np.array([0, 3]), parent=[-1, 0, 0], near=None, u=np.zeros(3, np.float32), u_next=np.array([.99], np.float32))
    got, nxt, _ = same(c, [0.0])
    assert got == [[0, 2]] and nxt == [17]


def test_long_sequences():
    """More drafts than a block has threads, as a chain that is taken far and as a broad tree."""
    V = 40
    x = np.zeros((1500, V), np.float32)
    tokens = np.arange(1500) % V
    for j in range(1499):
        x[j, tokens[j + 1]] = 9.0               # the target agrees with nearly every draft
    c = dict(x=torch.tensor(x, device="cuda"), tokens=tokens.tolist(), cu=np.array([0, 1400, 1500]), parent=None, near=None,
             u=np.random.default_rng(0).random(1500).astype(np.float32), u_next=np.array([.2, .8], np.float32))
    got, _, _ = same(c)
    c["u"][:] = 0.5
    got, _, _ = same(c)
    assert len(got[0]) == 1400 and len(got[1]) == 100
    got, _, _ = same(c, most=700)
    assert len(got[0]) == 700
    broad = case(5, 3000, [1300, 2], True, False, "f32")
    broad["parent"] = [-1] + [0] * 1299 + [-1, 0]
    same(broad)


def test_walks_that_end_early():
    c = case(2, 50, [9, 9, 9], False, False, "f32")
    c["u"][:] = 0
    for most in (1, 2, 5):
        got, _, _ = same(c, most=most)
        assert all(len(g) <= most for g in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_alignment(dtype):
    """Rows of any alignment, columns of wider arrays, both arrays."""
    V, add = 1003, [5, 4]
    c = case(8, V, add, True, True, dtype)
    wide = torch.full((9, V + 37), float("nan"), dtype=TYPES[dtype], device="cuda")
    near = torch.full((9, V + 11), float("nan"), device="cuda")
    for off in (1, 3, 8):
        wide[:, off:off + V] = c["x"]
        near[:, off:off + V] = torch.tensor(c["near"], device="cuda")
        same(c, x=wide[:, off:off + V], near=near[:, off:off + V])


def test_reported_and_passed_over():
    """Drafts with a parent or token out of range are passed over, a bad list counts as empty; the status says so once."""
    c = case(4, 100, [4, 4], True, False, "f32")
    for tokens, parent in (([1, -1, 2, 100, 1, 2, 3, 4], [-1, 0, 0, 0, -1, 0, 0, 0]), ([1, 2, 3, 4, 1, 2, 3, 4], [-1, 0, 2, -1, -1, 0, 7, 1])):
        c["tokens"], c["parent"] = tokens, parent
        c["u"][:] = 0.3
        got, nxt, _, v = run(c)
        want = ref.verify(c["x"].double().cpu().numpy(), tokens, c["cu"], c["u"], c["u_next"], [p if 0 <= p < j % 4 else -9 for j, p in enumerate(parent)], None, None, 4)
        assert got == want[0] and nxt == want[1]
        assert v.device_status() == 7 and v.device_status() == 0
    for cu in ([0, 4, 99], [0, 5, 4], [-1, 4, 8]):
        bad = dict(c, cu=np.array(cu), tokens=[1, 2, 3, 4] * 2, parent=[-1, 0, 0, 0] * 2)
        v = B.DraftVerifier(max_seqs=2, max_path=8, max_tokens=8)
        keep, n_keep, nxt = v.verify(bad["x"], ints(bad["tokens"]), ints(cu), floats(c["u"]), floats(c["u_next"]), parent=ints(bad["parent"]))
        broken = 0 if cu[0] < 0 else 1
        assert int(n_keep[broken]) == 0 and int(nxt[broken]) == -1 and (keep[broken] == -1).all()
        assert v.device_status() == 7


def test_lists_that_overlap():
    """A list that does not ascend: that sequence is empty, the others stay inside of their rows, whatever the workspace held before."""
    c = case(6, 64, [4, 4], True, True, "f32")
    for temperature in ([1.0] * 3, [0.0] * 3):
        v = B.DraftVerifier(max_seqs=3, max_path=8, max_tokens=8)
        v.workspace[256:] = 0x7f
        keep, n_keep, nxt = v.verify(c["x"], ints(c["tokens"]), ints([0, 5, 3, 8]), floats(c["u"]), floats([.1, .5, .9]), parent=ints([-1, 0, 0, 1, 1, -1, 0, 1]),
                                     draft_probs=torch.tensor(c["near"], device="cuda"), temperature=floats(temperature))
        assert n_keep.tolist()[1] == 0 and nxt.tolist()[1] == -1 and v.device_status() == 7
        assert all(-1 <= t < 64 for t in nxt.tolist()) and all(m >= 1 for m in n_keep.tolist()[::2])


def test_tokens_that_are_an_earlier_result():
    """Plain sampling may be given the object's own `next` as tokens; sequences of several rows then count as empty."""
    V, n = 500, 6
    c = case(9, V, [1] * n, False, False, "f32")
    v = B.DraftVerifier(max_seqs=n, max_path=2)
    _, want, _, _ = run(c, verifier=v)
    out = v.verify(c["x"], v.next, ints(range(n + 1)), floats(c["u"]), floats(c["u_next"]))
    assert out[2].tolist() == want and v.device_status() == 0
    out = v.verify(c["x"], v.next, ints([0, 2, 2, 3, 4, 5, 6]), floats(c["u"]), floats(c["u_next"]))
    assert out[1].tolist() == [0, 0, 1, 1, 1, 1] and out[2].tolist()[:2] == [-1, -1] and v.device_status() == 7
    with pytest.raises(Exception):
        v.verify(c["x"], ints([0] * n), v.keep.flatten()[:n + 1], floats(c["u"]), floats(c["u_next"]))


def test_no_rows():
    v = B.DraftVerifier(max_seqs=3, max_path=2)
    keep, n_keep, nxt = v.verify(torch.zeros((0, 10), device="cuda"), ints([]), ints([0, 0, 0, 0]), floats([]), floats([.1, .2, .3]))
    assert (keep == -1).all() and n_keep.tolist() == [0, 0, 0] and nxt.tolist() == [-1, -1, -1]


@pytest.mark.parametrize("tree", [False, True])
def test_tokens_follow_the_target(tree):
    """Over many uniform numbers the token behind the standing one is distributed as the target's own, whatever the drafter's is."""
    V, n, kids = 6, 60000, 3
    rng = np.random.default_rng(5)
    p, q = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V)).astype(np.float32)
    q64 = q.astype(np.float64) / q.astype(np.float64).sum()
    rows = 1 + (kids if tree else 1)
    x = torch.tensor(np.log(p), dtype=torch.float32, device="cuda").expand(n * rows, V)
    tokens = rng.choice(V, size=n * rows, p=q64)
    v = B.DraftVerifier(max_seqs=n, max_path=2, max_tokens=n * rows)
    keep, n_keep, nxt = v.verify(x.contiguous(), ints(tokens), ints(np.arange(n + 1) * rows), floats(rng.random(n * rows)), floats(rng.random(n)),
                                 parent=ints(([-1] + [0] * (rows - 1)) * n), draft_probs=torch.tensor(q, device="cuda").expand(n * rows, V).contiguous())
    keep, n_keep, nxt = keep.cpu().numpy(), n_keep.cpu().numpy(), nxt.cpu().numpy()
    first = np.where(n_keep > 1, tokens[np.arange(n) * rows + np.maximum(keep[:, 1], 0)], nxt)
    # each count is binomial: within 6 of its standard deviations (the numbers are fixed, so this holds always or never)
    count = np.bincount(first, minlength=V)
    assert (np.abs(count - n * p) <= 6 * np.sqrt(n * p * (1 - p)) + 1).all(), (count / n, p)


def test_repeated_calls_and_graph():
    """One object, different batches in turn, and a captured call that reads what its arrays hold then."""
    v = B.DraftVerifier(max_seqs=6, max_path=12, max_tokens=40)
    cases = [case(s, 2000, a, t, d, "bf16") for s, (a, t, d) in enumerate((([5, 1, 9, 0, 3, 12], True, False), ([1], False, True), ([9, 9], False, True)))]
    for c in cases + cases[::-1]:
        got, nxt, _, _ = run(c, verifier=v)
        want = ref.verify(c["x"].double().cpu().numpy(), c["tokens"], c["cu"], c["u"], c["u_next"], c["parent"], c["near"], None, 12)
        assert got == want[0] and nxt == want[1]
    c = cases[2]
    args = [c["x"], ints(c["tokens"]), ints(c["cu"]), floats(c["u"]), floats(c["u_next"])]
    near = torch.tensor(c["near"], device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = v.verify(*args, draft_probs=near)
        for seed in range(3):
            rng = np.random.default_rng(seed)
            u, u_next = rng.random(18).astype(np.float32), rng.random(2).astype(np.float32)
            args[3].copy_(floats(u))
            args[4].copy_(floats(u_next))
            graph.replay()
            want = ref.verify(c["x"].double().cpu().numpy(), c["tokens"], c["cu"], u, u_next, None, c["near"], None, 12)
            assert [k[:m] for k, m in zip(out[0].tolist(), out[1].tolist())] == want[0] and out[2].tolist() == want[1]


@pytest.mark.parametrize("best", [20.0, 40.0, 100.0, 2000.0, 1e4, -30.0])
@pytest.mark.parametrize("temperature", [1e-9, 2e-9, 1e-8, 1e-7, 1e-6, 1e-5, 1e-4])
def test_words_a_few_steps_below_the_best(best, temperature):
    """Small temperatures, where the steps of fp32 at the largest logit are as far apart as the powers of 2 that 64 bits hold: words 1 to 20 steps below
    it, as next tokens and as the rest beside a draft that 64 bits decide on."""
    n, V, best, temperature = 40, 60, np.float32(best), float(np.float32(temperature))
    below = [best]
    for _ in range(40):
        below.append(np.nextafter(below[-1], np.float32(-np.inf)))
    x = np.full((2 * n, V), best - np.float32(50), np.float32)
    for r in range(2 * n):
        x[r, 37] = best
        x[r, 5] = below[1 + r % 20]
        if r >= n:
            x[r, 50] = below[2 * (1 + r % 20)]
    rng = np.random.default_rng(0)
    u = np.where(np.arange(2 * n) % 3, np.float32(1 - 2.0 ** -24), rng.random(2 * n)).astype(np.float32)
    same(dict(x=torch.tensor(x, device="cuda"), tokens=[37] * (2 * n), cu=np.arange(n + 1) * 2, parent=None, near=None, u=u, u_next=rng.random(n).astype(np.float32)),
         [temperature] * n)


# What 64 bits leave of an exact probability here: 2e-13 of each word's power of 2, the same again for the sum that it is divided by, and a step of
# 2^-53 for each of some 10^4 additions.  A cumulated sum is off by no more than that altogether.
P64 = 1e-12


def drawn(r, u_next):
    """The tokens that a sum of r past u_next times all of it may mean, where cumulated sums are off by P64."""
    total = np.cumsum(r)
    goal = float(u_next) * total[-1]
    return [t for t in np.flatnonzero(r > -1) if total[t] >= goal - P64 and (total[t] - r[t]) <= goal + P64 and (r[t] > 0 or total[-1] < P64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,noise", [(300, 3e-7), (1000, 1e-7), (8000, 3e-7), (8000, 1e-6), (40000, 1e-6)])
def test_drafter_nearly_the_target(dtype, V, noise):
    """The drafter's probabilities are the target's but for a few steps of fp32, as those of the same model in another batch: after a refusal the rest
    is made of these differences alone."""
    rng = np.random.default_rng(V)
    n = 40
    x = torch.tensor(rng.standard_normal((3 * n, V)) * 2).to(TYPES[dtype])
    temperature = np.where(np.arange(n) % 2, np.float32(0.7), np.float32(1.0))
    near, tokens = np.zeros((3 * n, V), np.float32), []
    p = [ref.target(row, float(temperature[r // 3])) for r, row in enumerate(x.double().numpy())]
    for r in range(3 * n):
        near[r] = p[r] * (1 + rng.standard_normal(V) * noise)
    for s in range(n):
        over = near[3 * s] / p[3 * s]
        tokens += [0, int(np.argmax(over)), int(rng.choice(V, p=p[3 * s] / p[3 * s].sum()))]       # the first draft is refused
    u = np.where(np.arange(3 * n) % 3 == 1, np.float32(1 - 2.0 ** -24), rng.random(3 * n)).astype(np.float32)
    c = dict(x=x.cuda(), tokens=tokens, cu=np.arange(n + 1) * 3, parent=[-1, 0, 0] * n, near=near, u=u, u_next=rng.random(n).astype(np.float32))
    got, nxt, _, v = run(c, temperature)
    assert v.device_status() == 0
    for s in range(n):
        q = near[3 * s].astype(np.float64)
        r = np.maximum(p[3 * s] - q, 0)
        second, R = tokens[3 * s + 2], r.sum()
        border = abs(float(u[3 * s + 2]) * q[second] * R - r[second])
        taken = float(u[3 * s + 2]) * q[second] * R < r[second]
        assert got[s] == ([0, 2] if taken else [0]) or border < P64, (s, got[s], taken)
        r = p[3 * s + 2] if got[s] == [0, 2] else np.maximum(r - q * R, 0)
        assert nxt[s] in drawn(r, c["u_next"][s]), (s, nxt[s], got[s], drawn(r, c["u_next"][s]), R)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_last_word_of_the_rest(dtype):
    """u_next at its end: the last word with a rest, behind which all words lie a step of fp32 below the drafter's."""
    rng = np.random.default_rng(3)
    n, V = 300, 4096
    x = torch.tensor(rng.standard_normal((2 * n, V)) * 3).to(TYPES[dtype])
    temperature = rng.uniform(0.5, 1.5, n).astype(np.float32)
    near = np.zeros((2 * n, V), np.float32)
    for r, row in enumerate(x.double().numpy()):
        p = ref.target(row, float(temperature[r // 2]))
        near[r] = np.nextafter(p.astype(np.float32), np.float32(1))
        near[r, :V // 2] = p[:V // 2] * 0.999
        near[r, 0] = 2 * p[0]
    u_next = np.where(np.arange(n) % 2, np.float32(1), np.float32(1 - 2.0 ** -24)).astype(np.float32)
    c = dict(x=x.cuda(), tokens=[0] * (2 * n), cu=np.arange(n + 1) * 2, parent=None, near=near, u=np.full(2 * n, 1 - 2.0 ** -24, np.float32), u_next=u_next)
    got, nxt, _ = same(c, temperature)
    assert all(g == [0] for g in got) and all(t == V // 2 - 1 for t in nxt[1::2])


@pytest.mark.parametrize("dtype,V", [("f32", 8192), ("f32", 16384), ("bf16", 16384), ("bf16", 65536)])
def test_sums_that_end_between_groups(dtype, V):
    """Rows of eight equal parts and u_next at eighths: the sum to be passed ends with a part, where only the order of additions tells on which side of it."""
    rng = np.random.default_rng(V)
    rows, parts = 30, 8
    x = np.repeat(np.tile(rng.random((rows, V // parts)) * -3.0, (1, parts)), parts - 1, 0)
    n = len(x)
    u_next = np.tile(np.arange(1, parts) / parts, rows).astype(np.float32)
    c = dict(x=torch.tensor(x).to(TYPES[dtype]).cuda(), tokens=[0] * n, cu=np.arange(n + 1), parent=None, near=None, u=np.zeros(n, np.float32), u_next=u_next)
    _, nxt, _, _ = run(c)
    # (the lightest word has 1e-7 of the whole, 64 bits are off by 1e-12)
    for s, t in enumerate(nxt):
        end = (1 + s % (parts - 1)) * (V // parts)
        assert t in (end - 1, end), (s, t, end)


@pytest.mark.parametrize("u_next", [-1.0, -1e-30, -0.0, 1.0, 2.0, float("nan"), float("inf"), float("-inf")])
def test_numbers_outside_of_their_range(u_next):
    """Where a word is eligible one comes out: -1 says that there is none."""
    x = np.full((3, 3000), -np.inf)
    x[:, 1000:2000] = np.random.default_rng(0).standard_normal((3, 1000))
    c = dict(x=torch.tensor(x, dtype=torch.float32).cuda(), tokens=[0] * 3, cu=np.arange(4), parent=None, near=None, u=np.zeros(3, np.float32), u_next=np.full(3, u_next, np.float32))
    _, nxt, _, v = run(c)
    assert all(1000 <= t < 2000 for t in nxt) and v.device_status() == 0
