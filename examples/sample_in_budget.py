"""Sampled decoding with drafts over a cache of bounded size: path-composed MoE blocks of this library, attention with normed and
rotated heads, verification from random numbers, eviction by attention weight.

Prompts run packed and fill the cache; their last rows' attention says which positions matter.  Then, turn by turn, a small drafter
proposes a tree of tokens per sequence, one pass over the cache scores them, the walk that the random numbers take is kept, its
rows' attention is added to the positions' weights, and sequences that outgrow their budget lose the lightest positions.
Nothing between the calls waits for the host but the example's own drafter.  Weights are random; what the example shows is which
call does what.

    python examples/sample_in_budget.py
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


def floats(v):
    return torch.tensor(np.asarray(v, np.float32), device=DEV)


def cu_of(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]))


class Decoder:
    """Blocks of attention (grouped heads, normed and rotated, paged cache) and a path-composed MoE layer; bf16, random weights."""

    def __init__(self, blocks=2, hidden=256, heads=8, kv_heads=2, head_dim=64, vocab=500, max_tokens=512, max_seqs=4, page=16, max_len=512, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        draw = lambda *shape, fan: (torch.randn(shape, generator=g, device=DEV) / fan ** 0.5).bfloat16()
        self.heads, self.kv_heads, self.d, self.blocks, self.vocab = heads, kv_heads, head_dim, blocks, vocab
        self.embed = draw(vocab, hidden, fan=1.0)
        self.head = draw(hidden, vocab, fan=hidden / 9)
        self.w_qkv = [draw(hidden, (heads + 2 * kv_heads) * head_dim, fan=hidden) for _ in range(blocks)]
        self.w_out = [draw(heads * head_dim, hidden, fan=heads * head_dim) for _ in range(blocks)]
        inv_freq = 10000.0 ** (-np.arange(head_dim // 2) / (head_dim // 2))
        self.rotation, self.moe = [], []
        for b in range(blocks):
            self.rotation.append(B.HeadRotation(q_heads=heads, kv_heads=kv_heads, head_dim=head_dim, inv_freq=inv_freq, q_weight=1 + draw(head_dim, fan=16),
                                                k_weight=1 + draw(head_dim, fan=16)))
            cfg = wl.stack_layer_config(wl.small_case(seed, T=max_tokens, H=hidden, F=256, n=6, K=2), b)
            L = wl.make_layer(cfg)
            layer = B.PathMoELayer(n_experts=cfg.n, top_k=cfg.K, hidden=hidden, ffn=cfg.F, mask=L.mask, bias=L.bias, w_gate=B.to_device(L.w_gate),
                                   w_up=B.to_device(L.w_up), w_down=B.to_device(L.w_down), max_tokens=max_tokens)
            layer.set_router(B.to_device(wl.make_router_weights(cfg)[0]))
            self.moe.append(layer)
        self.attn = B.Attention(q_heads=heads, kv_heads=kv_heads, head_dim=head_dim, max_tokens=max_tokens, max_seqs=max_seqs)
        self.cache = B.PagedCache(layers=blocks, pages=max_seqs * (max_len // page), page_size=page, kv_heads=kv_heads, head_dim=head_dim, max_seqs=max_seqs,
                                  max_pages=max_len // page)
        self.weights = B.CacheWeights(self.cache, q_heads=heads)
        self.verifier = B.DraftVerifier(max_seqs=max_seqs, max_path=16, max_tokens=max_tokens)

    def run(self, tokens, position, seqs, cu, tree_mask=None, prompt=False):
        """One pass over packed tokens whose places in the cache are reserved.  Returns their logits and, block by block, what their
        attention leaves for weighing: queries and log sums."""
        norm = lambda x: torch.nn.functional.rms_norm(x, x.shape[-1:])
        h, left = self.embed[tokens.long()], []
        nq, nk = self.heads * self.d, self.kv_heads * self.d
        for b, layer in enumerate(self.moe):
            qkv = norm(h) @ self.w_qkv[b]                                             # a plain library product
            q, k, v = qkv[:, :nq].unflatten(1, (self.heads, self.d)), qkv[:, nq:nq + nk].unflatten(1, (self.kv_heads, self.d)), \
                qkv[:, nq + nk:].unflatten(1, (self.kv_heads, self.d))
            # over q and k themselves; a prompt's attention reads the packed keys, later ones the cache
            self.rotation[b].rotate_cached(q, k, v, position, self.cache, b, seqs, cu, k_out=k if prompt else None)
            lse = torch.empty((q.shape[0], self.heads), dtype=torch.float32, device=DEV)
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            if prompt:
                self.attn.prompt(q, k, v, cu, out, lse)
            else:
                self.attn.cached(q, self.cache, b, seqs, cu, tree_mask, out, lse)
            left.append((q, lse))
            h = h + out.flatten(1) @ self.w_out[b]
            layer.forward_hidden(norm(h))
            nxt = torch.empty_like(h)
            B.pcomoe_residual_cast(layer.layer, h.shape[0], h, layer.y, nxt)
            h = nxt
        return norm(h) @ self.head, left

    def weigh(self, left, seqs, cu, keep=None, n_keep=None):
        """The rows' attention into the positions' weights, all blocks together."""
        for b, (q, lse) in enumerate(left):
            self.weights.add(q, lse, b, seqs, cu, keep=keep, n_keep=n_keep, fresh=b == 0)


class Drafter:
    """Proposes from a table: a distribution of the next token for every token."""

    def __init__(self, vocab, rng):
        x = rng.standard_normal((vocab, vocab)) * 1.5
        self.p = np.exp(x) / np.exp(x).sum(1, keepdims=True)
        self.rng = rng

    def tree(self, first, shape=(2, 2, 1)):
        """A tree of drafts behind the token `first`, shape[i] children at depth i: tokens, parents."""
        tokens, parents, level = [int(first)], [-1], [0]
        for kids in shape:
            nxt = []
            for up in level:
                for t in self.rng.choice(len(self.p), size=kids, p=self.p[tokens[up]]):
                    tokens.append(int(t))
                    parents.append(up)
                    nxt.append(len(tokens) - 1)
            level = nxt
        return tokens, parents

    def rows(self, tokens):
        return floats(self.p[np.asarray(tokens)])


def ancestors(parents):
    bits = []
    for j, p in enumerate(parents):
        bits.append((1 << j) | (bits[p] if p >= 0 else 0))
    return bits


def depths(parents):
    out = []
    for p in parents:
        out.append(0 if p < 0 else out[p] + 1)
    return out


def generate(model, drafter, prompts, turns=12, budget=48, temperature=0.9, seed=0):
    """Returns the sequences and the lengths that the cache holds after each turn."""
    rng = np.random.default_rng(seed)
    n = len(prompts)
    seqs, lens = ints(range(n)), [len(p) for p in prompts]
    temp = floats([temperature] * n)
    u = lambda k: torch.tensor(rng.random(k).astype(np.float32), device=DEV)
    model.cache.reserve(seqs, ints(lens))
    cu = cu_of(lens)
    logits, left = model.run(ints(np.concatenate(prompts)), ints(np.concatenate([np.arange(k) for k in lens])), seqs, cu, prompt=True)
    model.weigh(left, seqs, cu)
    # the token behind each prompt: plain sampling, a sequence of one row each
    ends = torch.tensor(np.cumsum(lens) - 1, device=DEV)
    _, _, nxt = model.verifier.verify(logits[ends], ints([0] * n), cu_of([1] * n), u(n), u(n), temperature=temp)
    out, held = [list(p) + [int(t)] for p, t in zip(prompts, nxt.tolist())], []
    for _ in range(turns):
        trees = [drafter.tree(o[-1]) for o in out]
        counts = [len(t) for t, _ in trees]
        cu, flat = cu_of(counts), [t for tokens, _ in trees for t in tokens]
        parent = ints([p for _, parents in trees for p in parents])
        mask = torch.tensor(np.asarray([[b] for _, parents in trees for b in ancestors(parents)], np.uint32).view(np.int32), device=DEV)
        # a token's position is its place in the text, whatever the cache still holds of it
        position = ints([len(o) - 1 + d for o, (_, parents) in zip(out, trees) for d in depths(parents)])
        model.cache.reserve(seqs, ints(counts))
        logits, left = model.run(ints(flat), position, seqs, cu, mask)
        keep, n_keep, nxt = model.verifier.verify(logits, ints(flat), cu, u(len(flat)), u(n), parent=parent, draft_probs=drafter.rows(flat), temperature=temp)
        model.cache.keep(seqs, cu, keep, n_keep)
        model.weigh(left, seqs, cu, keep, n_keep)
        model.weights.evict(seqs, ints([budget] * n), sinks=2, recent=16)
        for i, (path, m, t) in enumerate(zip(keep.tolist(), n_keep.tolist(), nxt.tolist())):
            out[i] += [trees[i][0][j] for j in path[1:m]] + [t]
        held.append(model.cache.seq_len[:n].tolist())
    return out, held


def main():
    model = Decoder()
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, model.vocab, size=k).tolist() for k in (37, 5, 64)]
    out, held = generate(model, Drafter(model.vocab, rng), prompts)
    print("tokens after 12 turns:", [len(o) - len(p) for o, p in zip(out, prompts)], "held in the cache:", held[-1])
    status = [model.cache.device_status(), model.attn.device_status(), model.weights.device_status(), model.verifier.device_status()]
    assert status == [0, 0, 0, 0], status
    return model, prompts, out, held


if __name__ == "__main__":
    main()
