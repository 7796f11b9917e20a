"""Speculative decoding of a small verifier whose keys and values are cached in 4 bits.

    python examples/verify_with_cache.py [--steps 24]

Every layer of a random-weight decoder keeps a KvCache.  A prompt enters in
causal chunks; then each step drafts a tree from the semantic pool, verifies it
in one forward (attend under the tree's mask, the nodes' own keys and values
beside the cached ones), walks the accepted path, adds up the attention weight
its rows gave (weigh), commits their keys and values (append) and brings every
head back to its budget (evict).  Nothing in a step waits for the host.

The decoder's head favours one successor per token, so that stored traffic
predicts it and drafts are accepted.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import torch

import paper_2608_03839_amd as oil

CHUNK = 256


class Verifier:
    """A decoder of attention layers alone, weights from the seed."""

    def __init__(self, requests, capacity, layers=2, width=256, q_heads=8, heads=2, head_dim=64, vocab=997, seed=0,
                 device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        bf16 = dict(device=device, dtype=torch.bfloat16)
        normal = lambda *shape: torch.randn(shape, generator=g, device=device)  # noqa: E731
        self.shape = (q_heads, heads, head_dim)
        self.embedding = normal(vocab, width).to(**bf16)
        self.successor = torch.randperm(vocab, generator=g, device=device)
        # logits of token t: what follows t is the row that looks like t
        self.head = torch.empty_like(self.embedding)
        self.head[self.successor] = self.embedding
        self.rate = torch.exp(-torch.arange(0, head_dim, 2, device=device) * (math.log(1e4) / head_dim))
        columns = (q_heads + 2 * heads) * head_dim
        self.qkv = [(normal(width, columns) / math.sqrt(width)).to(**bf16) for _ in range(layers)]
        self.out = [(0.3 * normal(q_heads * head_dim, width) / math.sqrt(q_heads * head_dim)).to(**bf16)
                    for _ in range(layers)]
        self.caches = [oil.KvCache(requests, heads, head_dim, capacity, device=device) for _ in range(layers)]

    def _turn(self, x, position):
        """Rotary encoding of x (B, N, heads, dim) at position (B, N)."""
        angle = position[:, :, None, None] * self.rate
        even, odd = x[..., 0::2].float(), x[..., 1::2].float()
        return torch.stack([even * angle.cos() - odd * angle.sin(), even * angle.sin() + odd * angle.cos()],
                           -1).flatten(3).to(x.dtype)

    def forward(self, tokens, position, n_nodes=None, mask=None):
        """Nodes (B, N) over the caches -> states (B, N, width), predictions (B, N) and, for each
        layer, what its cache is given afterwards."""
        q_heads, heads, dim = self.shape
        B, N = tokens.shape
        x, kept = self.embedding[tokens], []
        for qkv, out, cache in zip(self.qkv, self.out, self.caches):
            heads_of = torch.matmul(x, qkv).view(B, N, q_heads + 2 * heads, dim)
            heads_of[:, :, :q_heads + heads] = self._turn(heads_of[:, :, :q_heads + heads], position)
            q, k, v = heads_of.split([q_heads, heads, heads], dim=2)  # views of one buffer
            o, lse = cache.attend(q, k, v, n_nodes=n_nodes, mask=mask)
            x = x + torch.matmul(o.view(B, N, -1), out)
            kept.append((q, k, v, lse))
        return x, torch.matmul(x, self.head.T).argmax(-1).to(torch.int32), kept


def run(requests=3, prompt=300, steps=24, keep=320, recent=64, seed=0, device="cuda"):
    """-> (accepted nodes of each step (steps, requests), the verifier)."""
    dev = torch.device(device)
    nodes = 1 + 16
    model = Verifier(requests, keep + nodes, seed=seed, device=dev)
    width = model.embedding.shape[1]
    g = torch.Generator(device=dev)
    g.manual_seed(seed + 1)
    # prompts of successors, each begun anew every 50 tokens
    tokens = torch.randint(model.embedding.shape[0], (requests, prompt), generator=g, device=dev)
    for i in range(1, prompt):
        if i % 50:
            tokens[:, i] = model.successor[tokens[:, i - 1]]
    pool = oil.Pool(width, requests * prompt, device=dev)
    x = None
    for i in range(0, prompt, CHUNK):
        chunk = tokens[:, i:i + CHUNK].contiguous()
        position = torch.arange(i, i + chunk.shape[1], device=dev).expand(requests, -1)
        x, _, kept = model.forward(chunk, position)
        for cache, (q, k, v, lse) in zip(model.caches, kept):
            cache.append(k, v)
            cache.evict(keep, recent)
        for b in range(requests):
            trace = torch.full((chunk.shape[1],), b, dtype=torch.int32, device=dev)
            pool.append(x[b].contiguous(), chunk[b].to(torch.int32), trace, trace)
    # a step's query is the state of its anchor's predecessor, as stored states are of theirs
    state, anchor = x[:, -2].contiguous(), tokens[:, -1].to(torch.int32)
    last = torch.full((requests,), prompt - 1, device=dev)
    rule = oil.DepthRule.fixed(8, theta=0.5)
    accepted, at = [], torch.arange(requests, device=dev)
    for step in range(steps):
        scores, idx = pool.query_topk(state, 4)
        chains, lengths = pool.gather(idx, scores, rule, 8)
        node_token, node_parent, _, n_nodes = oil.merge_trees(anchor, None, None, 0, chains, lengths, nodes - 1, nodes)
        mask = oil.tree_mask(node_parent, n_nodes)
        words = mask.to(torch.int64) & 0xFFFFFFFF
        depth = ((words[..., None] >> torch.arange(32, device=dev)) & 1).sum((-1, -2)) - 1
        x, target, kept = model.forward(node_token.clamp(min=0).long(), last[:, None] + depth.clamp(min=0), n_nodes, mask)
        accept_len, accept_nodes, bonus = oil.accept_walk(node_token, node_parent, n_nodes, target)
        for cache, (q, k, v, lse) in zip(model.caches, kept):
            cache.weigh(q, lse, nodes=accept_nodes, count=accept_len)
            cache.append(k, v, nodes=accept_nodes, count=accept_len)
            cache.evict(keep, recent)
        # the state before the next anchor is that of the last node committed
        end = torch.where(accept_len > 0, accept_nodes[at, (accept_len - 1).clamp(min=0).long()], 0).long()
        state, anchor, last = x[at, end].contiguous(), bonus, last + accept_len + 1
        accepted.append(accept_len)
    return torch.stack(accepted), model


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=24)
    a = ap.parse_args()
    accepted, model = run(steps=a.steps)
    print(f"accepted nodes a step: {accepted.float().mean().item():.2f}")
    for i, cache in enumerate(model.caches):
        print(f"layer {i}: {cache.lengths.tolist()} rows held of {cache.state[:, 1].tolist()} positions, "
              f"heaviest weight {cache.weights.amax().item():.1f}")


if __name__ == "__main__":
    main()
