"""Drafted decoding with a small random decoder: path-composed MoE blocks of this library with attention in front of them.

Prompts of different lengths are run packed and fill a paged cache; then, turn by turn, a tree of drafted tokens per sequence
is verified in one pass over the cache, the accepted branch is kept and the rest rolled back.  One sequence is forked on
the way and compared with its parent, and the pool is compacted at the end.  Weights and drafts are random (a real drafter
proposes better); what the example shows is which call does what, and it checks the drafted turns against one packed pass over
the whole sequences.

    python examples/draft_and_verify.py
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2609_01024_b200 import binding as B  # noqa: E402
from paper_2609_01024_b200 import workloads as wl  # noqa: E402

DEV = "cuda:0"


def ints(v):
    return torch.tensor(np.asarray(v, np.int32), device=DEV)


def cu_of(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]))


class Decoder:
    """Blocks of attention (grouped heads, paged cache) and a path-composed MoE layer; bf16, random weights."""

    def __init__(self, blocks=2, hidden=256, heads=8, kv_heads=2, head_dim=64, vocab=1000, max_tokens=512, max_seqs=8, page=16,
                 max_len=512, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        draw = lambda *shape, fan: (torch.randn(shape, generator=g, device=DEV) / fan ** 0.5).bfloat16()
        self.heads, self.kv_heads, self.d = heads, kv_heads, head_dim
        self.embed = draw(vocab, hidden, fan=1.0)
        self.head = draw(hidden, vocab, fan=hidden)
        self.w_qkv = [draw(hidden, (heads + 2 * kv_heads) * head_dim, fan=hidden) for _ in range(blocks)]
        self.w_out = [draw(heads * head_dim, hidden, fan=heads * head_dim) for _ in range(blocks)]
        self.moe = []
        for b in range(blocks):
            cfg = wl.stack_layer_config(wl.small_case(seed, T=max_tokens, H=hidden, F=256, n=6, K=2), b)
            L = wl.make_layer(cfg)
            layer = B.PathMoELayer(n_experts=cfg.n, top_k=cfg.K, hidden=hidden, ffn=cfg.F, mask=L.mask, bias=L.bias,
                                   w_gate=B.to_device(L.w_gate), w_up=B.to_device(L.w_up), w_down=B.to_device(L.w_down), max_tokens=max_tokens)
            layer.set_router(B.to_device(wl.make_router_weights(cfg)[0]))
            self.moe.append(layer)
        self.attn = B.Attention(q_heads=heads, kv_heads=kv_heads, head_dim=head_dim, max_tokens=max_tokens, max_seqs=max_seqs)
        pages = max_seqs * (max_len // page)
        self.cache = B.PagedCache(layers=blocks, pages=pages, page_size=page, kv_heads=kv_heads, head_dim=head_dim, max_seqs=max_seqs,
                                  max_pages=max_len // page)
        self.scores = B.TokenScores(max_tokens=max_tokens, top_n=3)

    def run(self, tokens, attend):
        """Hidden states -> logits of packed tokens.  attend(block, q, k, v) -> the block's attention output."""
        norm = lambda x: torch.nn.functional.rms_norm(x, x.shape[-1:])
        h = self.embed[tokens.long()]
        nq, nk = self.heads * self.d, self.kv_heads * self.d
        for b, layer in enumerate(self.moe):
            qkv = norm(h) @ self.w_qkv[b]                                             # a plain library product
            q, k, v = qkv[:, :nq].unflatten(1, (self.heads, self.d)), qkv[:, nq:nq + nk].unflatten(1, (self.kv_heads, self.d)), \
                qkv[:, nq + nk:].unflatten(1, (self.kv_heads, self.d))
            h = h + attend(b, q, k, v).flatten(1) @ self.w_out[b]
            layer.forward_hidden(norm(h))
            out = torch.empty_like(h)
            B.pcomoe_residual_cast(layer.layer, h.shape[0], h, layer.y, out)
            h = out
        return norm(h) @ self.head

    def prompt(self, tokens, cu, seqs=None, lens=None):
        """Packed prompts; with `seqs` their keys and values go into the cache."""
        if seqs is not None:
            self.cache.reserve(seqs, lens)

        def attend(b, q, k, v):
            if seqs is not None:
                self.cache.write(k, v, seqs, cu, layer=b)
            return self.attn.prompt(q, k, v, cu)[0]
        return self.run(tokens, attend)

    def verify(self, tokens, cu, seqs, counts, tree_mask):
        """One pass over drafted tokens: every row sees the context and its own ancestors."""
        self.cache.reserve(seqs, counts)

        def attend(b, q, k, v):
            self.cache.write(k, v, seqs, cu, layer=b)
            return self.attn.cached(q, self.cache, b, seqs, cu, tree_mask)[0]
        return self.run(tokens, attend)


def draft_tree(rng, first, vocab, n):
    """n drafted tokens, the first one given (number 0), the others random words behind random earlier ones: (tokens, parents)."""
    parents = [-1] + [int(rng.integers(0, j)) for j in range(1, n)]
    return [int(first)] + rng.integers(0, vocab, size=n - 1).tolist(), parents


def ancestors(parents):
    bits = []
    for j, p in enumerate(parents):
        bits.append((1 << j) | (bits[p] if p >= 0 else 0))
    return bits


def generate(model, prompts, turns=6, drafts=30, seed=1):
    """Greedy drafted decoding.  Returns the sequences and, per accepted token, its log probability and entropy."""
    rng = np.random.default_rng(seed)
    vocab = model.head.shape[1]
    n = len(prompts)
    lens, seqs = [len(p) for p in prompts], ints(range(n))
    logits = model.prompt(ints(np.concatenate(prompts)), cu_of(lens), seqs, ints(lens))
    last = logits[torch.tensor(np.cumsum(lens) - 1, device=DEV)].contiguous()
    _, _, ids, _ = model.scores.score(last, ints([-1] * n))
    nxt = ids[:, 0].tolist()
    out, told = [list(p) for p in prompts], [[] for _ in range(n)]
    for _ in range(turns):
        trees = [draft_tree(rng, nxt[i], vocab, drafts) for i in range(n)]
        flat = ints([t for tree, _ in trees for t in tree])
        counts = [len(tree) for tree, _ in trees]
        cu = cu_of(counts)
        mask = torch.tensor(np.asarray([[b] for _, parents in trees for b in ancestors(parents)], np.uint32).view(np.int32), device=DEV)
        logits = model.verify(flat, cu, seqs, ints(counts), mask)
        # the score of every drafted token is read at its parent's row; the first one was the best already
        parent_row = np.concatenate([[0 if p < 0 else p for p in parents] + np.int64(sum(counts[:i])) for i, (_, parents) in enumerate(trees)])
        lp, ent, ids, _ = model.scores.score(logits[torch.tensor(parent_row, device=DEV)].contiguous(), flat)
        lp, ent, best = lp.tolist(), ent.tolist(), ids[:, 0].tolist()               # best[j]: the best word behind j's parent
        _, _, own_best, _ = model.scores.score(logits, ints([-1] * flat.numel()))
        own = own_best[:, 0].tolist()
        keep = []
        for i, (tokens, parents) in enumerate(trees):
            at, path = sum(counts[:i]), [0]
            while True:                                                               # the child that is the best word, if drafted
                kids = [j for j in range(len(tokens)) if parents[j] == path[-1] and best[at + j] == tokens[j]]
                if not kids:
                    break
                path.append(kids[0])
            keep.append(path)
            out[i] += [tokens[j] for j in path]
            told[i] += [(lp[at + j], ent[at + j]) for j in path[1:]]
            nxt[i] = own[at + path[-1]]
        width = max(len(p) for p in keep)
        model.cache.keep(seqs, cu, ints([p + [-1] * (width - len(p)) for p in keep]), ints([len(p) for p in keep]))
    return out, told, nxt


def main():
    model = Decoder(vocab=32)                  # few words, so that random drafts are accepted now and then
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, 32, size=k).tolist() for k in (37, 5, 64)]
    out, told, nxt = generate(model, prompts)
    kept = [len(o) - len(p) for o, p in zip(out, prompts)]
    print("tokens accepted per sequence in 6 turns:", kept)

    # the cache holds exactly the accepted sequences: the next word from it is the next word of one packed pass over them
    lens = [len(o) for o in out]
    assert model.cache.seq_len[:3].tolist() == lens
    whole = model.prompt(ints(np.concatenate(out)), cu_of(lens))[torch.tensor(np.cumsum(lens) - 1, device=DEV)]
    # best-of-n: a fork shares its pages until it grows; both then score their next token over the cache
    model.cache.fork(ints([0]), ints([5]))
    seqs = ints([0, 1, 2, 5])
    step = model.verify(ints(nxt + [nxt[0]]), cu_of([1] * 4), seqs, ints([1] * 4), None)
    again = model.prompt(ints(np.concatenate([o + [x] for o, x in zip(out, nxt)])), cu_of([k + 1 for k in lens]))
    again = again[torch.tensor(np.cumsum([k + 1 for k in lens]) - 1, device=DEV)]
    rel = float((step[:3].float() - again.float()).norm() / again.float().norm())
    print("next-token logits over the cache against one packed pass: relative difference %.4f" % rel)
    assert torch.equal(step[0], step[3]), "a fork and its parent see the same"
    used = int((model.cache.page_ref > 0).sum())
    model.cache.trim(ints([1, 5]), ints([0, 0]))
    model.cache.compact()
    left = int((model.cache.page_ref > 0).sum())
    print("pages in use: %d, after freeing two sequences and compacting: %d, the highest one number %d" %
          (used, left, int(model.cache.page_table.max())))
    assert int(model.cache.page_table.max()) == left - 1
    status = [model.cache.device_status(), model.attn.device_status()]
    assert status == [0, 0], status
    return rel, whole


if __name__ == "__main__":
    main()
