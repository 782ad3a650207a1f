"""Rotation, attention over the cache, verification, kept rows, weights and eviction together, as a serving loop runs them."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import turn_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("sample_in_budget", os.path.join(ROOT, "examples", "sample_in_budget.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_sampling_in_a_budget():
    m = example()
    model, prompts, out, held = m.main()
    for o, p in zip(out, prompts):
        assert o[:len(p)] == p and len(o) >= len(p) + 13 and all(0 <= t < model.vocab for t in o)
    assert all(k <= 48 for row in held for k in row) and max(held[-1]) == 48
    pages = sum(-(-k // model.cache.page_size) for k in held[-1])
    assert int((model.cache.page_ref > 0).sum()) == pages


def test_one_turn_step_by_step():
    """Every step of a turn against plain forms of the step before: cached keys, the walk, the weights, what is evicted."""
    m = example()
    B = m.B
    model, rng = m.Decoder(blocks=1, seed=3), np.random.default_rng(3)
    prompt = rng.integers(0, model.vocab, size=70).tolist()
    seqs = m.ints([0])
    model.cache.reserve(seqs, m.ints([70]))
    cu = m.cu_of([70])
    logits, left = model.run(m.ints(prompt), m.ints(range(70)), seqs, cu, prompt=True)
    model.weigh(left, seqs, cu)
    # every row's attention adds up to one a head
    total = float(model.weights.weight[0, :70].double().sum())
    assert abs(total - 70 * model.heads) <= 2e-5 * total
    drafter = m.Drafter(model.vocab, rng)
    tokens, parents = drafter.tree(5, (3, 2, 1))
    n = len(tokens)
    cu = m.cu_of([n])
    mask = torch.tensor(np.asarray([[b] for b in m.ancestors(parents)], np.uint32).view(np.int32), device="cuda")
    model.cache.reserve(seqs, m.ints([n]))
    logits, left = model.run(m.ints(tokens), m.ints([70 + d for d in m.depths(parents)]), seqs, cu, mask)
    u, u_next = rng.random(n).astype(np.float32), rng.random(1).astype(np.float32)
    near = drafter.rows(tokens)
    keep, n_keep, nxt = model.verifier.verify(logits, m.ints(tokens), cu, m.floats(u), m.floats(u_next), parent=m.ints(parents), draft_probs=near)
    path, want = ref.verify(logits.double().cpu().numpy(), tokens, [0, n], u, u_next, parents, near.cpu().numpy())
    assert keep[0, :int(n_keep[0])].tolist() == path[0] and nxt.tolist() == want
    model.cache.keep(seqs, cu, keep, n_keep)
    before = model.weights.weight[0].double().cpu().numpy()
    model.weigh(left, seqs, cu, keep, n_keep)
    length, base = int(model.cache.seq_len[0]), 70
    assert length == base + len(path[0])
    k = ref.rows_of(model.cache.k[0], model.cache.page_table[0].tolist(), model.cache.page_size, length).double().cpu().numpy()
    q, lse = left[0][0].double().cpu().numpy(), left[0][1].double().cpu().numpy()
    add, err = ref.weigh(q, lse, k, model.d ** -0.5, path[0], base)
    got = model.weights.weight[0, :length].double().cpu().numpy()
    old = np.concatenate([before[:base], np.zeros(length - base)])
    assert (np.abs(got - old - add) <= err + (old + add) * 2.0 ** -23).all()
    # the log sums came from the attention over the tree, which saw these positions alone: the kept rows' weights add up to one a head
    assert abs(float(add.sum()) - len(path[0]) * model.heads) <= 2e-5 * len(path[0]) * model.heads
    stays = ref.evict(got, length, 40, 2, 10)
    kept = torch.tensor(k)[stays]
    model.weights.evict(seqs, m.ints([40]), sinks=2, recent=10)
    assert int(model.cache.seq_len[0]) == 40
    now = ref.rows_of(model.cache.k[0], model.cache.page_table[0].tolist(), model.cache.page_size, 40).double().cpu()
    assert torch.equal(now, kept)
    assert [model.cache.device_status(), model.attn.device_status(), model.weights.device_status(), model.verifier.device_status()] == [0] * 4


def test_two_objects_at_the_same_time():
    """Two loops' objects on two streams, their calls interleaved, give what each gives alone."""
    m = example()
    B = m.B
    rng = np.random.default_rng(7)
    work = []
    for i, (V, rows, lens) in enumerate(((3000, 7, [900, 40]), (32000, 4, [60, 2500]))):
        n = len(lens)
        T = n * rows
        c = ref.cache_of(B, B.PCOMOE_BF16, page=16, kv_heads=2, head_dim=64, lens=lens, seed=i)
        w = dict(logits=torch.randn(T, V, device="cuda").bfloat16(), tokens=m.ints(rng.integers(0, V, T)), cu=m.cu_of([rows] * n), u=m.floats(rng.random(T)),
                 u_next=m.floats(rng.random(n)), near=torch.softmax(torch.randn(T, V, device="cuda"), 1), seqs=m.ints(range(n)), cache=c, weights=B.CacheWeights(c, q_heads=8),
                 q=torch.randn(T, 8, 64, device="cuda").bfloat16(), lse=torch.full((T, 8), 6.0, device="cuda"), verifier=B.DraftVerifier(max_seqs=n, max_path=rows),
                 rotation=B.HeadRotation(q_heads=8, kv_heads=2, head_dim=64, inv_freq=np.linspace(1, 0.001, 32)), k=torch.randn(T, 2, 64, device="cuda").bfloat16(),
                 position=m.ints(rng.integers(0, 9999, T)), stream=torch.cuda.Stream())
        work.append(w)

    def turn(w):
        w["weights"].weight.zero_()
        q = torch.empty_like(w["q"])
        w["rotation"].rotate_cached(w["q"], w["k"], w["k"], w["position"], w["cache"], 0, w["seqs"], w["cu"], q)
        out = [x.clone() for x in w["verifier"].verify(w["logits"], w["tokens"], w["cu"], w["u"], w["u_next"], draft_probs=w["near"])]
        w["weights"].add(q, w["lse"], 0, w["seqs"], w["cu"], fresh=True)
        return out + [q, w["weights"].weight.clone()]

    want = [turn(w) for w in work]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, w in enumerate(work):
            with torch.cuda.stream(w["stream"]):
                got[i] = turn(w)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert [w[k].device_status() for w in work for k in ("cache", "weights", "verifier")] == [0] * 6
