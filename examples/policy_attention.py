"""A policy's attention around the quantized projections, at the workloads' widths with random weights:

  1. the language layers read 816 prefix tokens: W4A4 q|k|v projection, head norms, rotation and an append to an 8-bit
     cache in one call, causal attention over the cache, W8A8 output projection;
  2. the action expert denoises 50 action tokens: its layers append them behind the prefix (the same slots at every
     step) and attend to everything in the cache, every token seeing every other;
  3. a second expert reads the language states by cross attention (keys and values projected once for all steps).

    python examples/policy_attention.py [--layers 2] [--steps 4] [--prefix 816] [--actions 50]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_24433_amd import fq  # noqa: E402


class CachedLayer:
    """q|k|v projection -> norm, rotation, append -> attention over the cache -> output projection, with a residual."""

    def __init__(self, width, heads, kv_heads, head_dim, gen, block=128):
        n = (heads + 2 * kv_heads) * head_dim
        self.heads, self.kv_heads, self.head_dim, self.width = heads, kv_heads, head_dim, width
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda") * 0.02  # noqa: E731
        self.qkv = fq.QuantLinear(rand(n, width), block, 4)
        self.o = fq.QuantLinear(rand(width, heads * head_dim), block, 8)
        self.q_norm, self.k_norm = (1.0 + rand(head_dim) for _ in range(2))

    def __call__(self, x, cache, batch, rope, max_new, max_kv, causal):
        pages, q_start, kv_len = batch
        h = self.qkv(x).view(x.shape[0], self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = h.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        q = fq.cache_append(cache, pages, q_start, kv_len, max_new, k, v, q, rope, q_weight=self.q_norm, k_weight=self.k_norm)
        a = fq.cache_attention(q, cache, pages, q_start, kv_len, max_new, max_kv, causal=causal)
        return x + self.o(a.view(x.shape[0], self.heads * self.head_dim))


class CrossLayer:
    """Queries from the action tokens, keys and values from the language states."""

    def __init__(self, width, state_width, heads, head_dim, gen, block=128):
        self.heads, self.head_dim = heads, head_dim
        rand = lambda *s: torch.randn(s, generator=gen, device="cuda") * 0.02  # noqa: E731
        self.q = fq.QuantLinear(rand(heads * head_dim, width), block, 4)
        self.kv = fq.QuantLinear(rand(2 * heads * head_dim, state_width), block, 4)
        self.o = fq.QuantLinear(rand(width, heads * head_dim), block, 8)

    def states(self, x):
        return self.kv(x).view(1, x.shape[0], 2 * self.heads, self.head_dim).chunk(2, dim=2)

    def __call__(self, x, states, mask=None):
        q = self.q(x).view(1, x.shape[0], self.heads, self.head_dim)
        a = fq.cross_attention(q, *states, key_mask=mask)
        return x + self.o(a.view(x.shape[0], self.heads * self.head_dim))


def run(layers=2, steps=4, prefix=816, actions=50, page=64, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    total = prefix + actions
    per_seq = -(-total // page)
    # the language model's heads and the expert's share a cache: 8 query heads on one key head of 256
    language = [CachedLayer(2048, 8, 1, 256, gen) for _ in range(layers)]
    expert = [CachedLayer(1024, 8, 1, 256, gen) for _ in range(layers)]
    cross = CrossLayer(1024, 2048, 16, 64, gen)
    caches = [fq.kv_cache(per_seq, 1, page, 256) for _ in range(layers)]
    inv_freq, magnitude = fq.rope_frequencies(256)
    rope = fq.rope_table(total, inv_freq, magnitude)
    pages = torch.randperm(per_seq, generator=gen, device="cuda").to(torch.int32)[None]
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731

    x = torch.randn((prefix, 2048), generator=gen, device="cuda").to(torch.bfloat16)
    batch = (pages, ints(0, prefix), ints(prefix))
    for layer, cache in zip(language, caches):
        x = layer(x, cache, batch, rope, prefix, prefix, True)
    states = cross.states(x)
    mask = torch.rand((1, prefix), generator=gen, device="cuda") < 0.9  # places of absent camera images are unseen

    y = torch.randn((actions, 1024), generator=gen, device="cuda").to(torch.bfloat16)
    batch = (pages, ints(0, actions), ints(total))
    for _ in range(steps):
        z = y
        for layer, cache in zip(expert, caches):
            z = layer(z, cache, batch, rope, actions, total, False)
        z = cross(z, states, mask)
        y = y - z / steps
    return y, x, caches, pages


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("layers", 2), ("steps", 4), ("prefix", 816), ("actions", 50)):
        ap.add_argument(f"--{name}", type=int, default=default)
    a = ap.parse_args()
    y, x, caches, _ = run(a.layers, a.steps, a.prefix, a.actions)
    torch.cuda.synchronize()
    held = sum(t.numel() * t.element_size() for c in caches for t in c)
    print(f"prefix {a.prefix} tokens, {a.steps} steps of {a.actions} action tokens, {a.layers} layers each: "
          f"actions rms {y.float().square().mean().sqrt().item():.4f}, cache {held / 1e6:.2f} MB")


if __name__ == "__main__":
    main()
