"""A policy's attention around the quantized projections, at the workloads' widths with random weights:

  1. the language layers read 816 prefix tokens: W4A4 q|k|v projection, head norms, rotation and an append to an 8-bit
     cache in one call, causal attention over the cache, W8A8 output projection;
  2. the action expert denoises 50 action tokens: its layers append them behind the prefix (the same slots at every
     step, the first of them in a copy of the prefix's last page) and attend to everything in the cache, every token
     seeing every other;
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


class Policy:
    """A prompt read once into the caches, then denoising steps over it.

    An append to a page that is in use may raise the page's scale, which rounds the earlier tokens' codes again, and a page
    given a value that is not finite is lost as a whole.  The steps write the same slots over and over, the first of them
    behind the prompt's last tokens: their page is a copy, made anew at every step, and the prompt's own stays as it was read."""

    def __init__(self, layers, prefix, actions, page, gen):
        total = prefix + actions
        per_seq = -(-total // page)
        self.prefix, self.actions = prefix, actions
        # the language model's heads and the expert's share a cache: 8 query heads on one key head of 256
        self.language = [CachedLayer(2048, 8, 1, 256, gen) for _ in range(layers)]
        self.expert = [CachedLayer(1024, 8, 1, 256, gen) for _ in range(layers)]
        self.cross = CrossLayer(1024, 2048, 16, 64, gen)
        self.caches = [fq.kv_cache(per_seq + 1, 1, page, 256) for _ in range(layers)]
        inv_freq, magnitude = fq.rope_frequencies(256)
        self.rope = fq.rope_table(total, inv_freq, magnitude)
        order = torch.randperm(per_seq + 1, generator=gen, device="cuda").to(torch.int32)
        self.pages, self.step_pages = order[None, :per_seq].contiguous(), order[None, :per_seq].clone()
        self.shared = None  # (the prompt's last page, the steps' copy of it)
        if prefix % page:
            self.shared = int(order[prefix // page]), int(order[per_seq])
            self.step_pages[0, prefix // page] = order[per_seq]
        ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.prompt_batch = (self.pages, ints(0, prefix), ints(prefix))
        self.step_batch = (self.step_pages, ints(0, actions), ints(total))

    def read(self, x, mask=None):
        """The prompt's tokens through the language layers; mask: the places that the second expert sees."""
        for layer, cache in zip(self.language, self.caches):
            x = layer(x, cache, self.prompt_batch, self.rope, self.prefix, self.prefix, True)
        self.states, self.mask = self.cross.states(x), mask
        return x

    def velocity(self, y):
        """One step's direction for the actions y."""
        z = y
        for layer, cache in zip(self.expert, self.caches):
            if self.shared is not None:
                kept, copy = self.shared
                for t in cache:
                    t[copy] = t[kept]
            z = layer(z, cache, self.step_batch, self.rope, self.actions, self.prefix + self.actions, False)
        return self.cross(z, self.states, self.mask)


def run(layers=2, steps=4, prefix=816, actions=50, page=64, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    policy = Policy(layers, prefix, actions, page, gen)
    x = torch.randn((prefix, 2048), generator=gen, device="cuda").to(torch.bfloat16)
    # places of absent camera images are unseen
    x = policy.read(x, torch.rand((1, prefix), generator=gen, device="cuda") < 0.9)
    y = torch.randn((actions, 1024), generator=gen, device="cuda").to(torch.bfloat16)
    for _ in range(steps):
        y = y - policy.velocity(y) / steps
    return y, x, policy.caches, policy.pages


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
