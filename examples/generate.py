#!/usr/bin/env python3
"""A transformer block that generates: attention over a paged 8-bit key/value cache, then the routed MoE feed-forward layer.

Prompts of different lengths go in as one chunk each, then every sequence takes one token at a time; random weights stand in for a model, and a
step's output row is the next step's input.

    python examples/generate.py [--seqs 16] [--prompt 300] [--tokens 32] [--bf16-cache] [--pictures]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2508_02317_amd import libmoe as L
from paper_2508_02317_amd.generation import CachedAttention, PagedKVCache, rope_axes, rope_frequencies
from paper_2508_02317_amd.layer import MoELayer


class Block:
    """x + attention(norm(x)), then + moe(norm(.)): one block of a decoder, weights N(0, 0.02)."""

    def __init__(self, d, heads, kv_heads, dim, experts, k, f, pages, page_size, n_pos, eight_bit=True, seed=0, sections=None, **scaling):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        mk = lambda *s: (torch.randn(s, generator=gen, device="cuda") * 0.02).bfloat16()
        self.d, self.experts, self.k, self.f = d, experts, k, f
        self.w_qkv, self.w_out, self.w_router = mk((heads + 2 * kv_heads) * dim, d), mk(d, heads * dim), mk(experts, d)
        self.w_gate, self.w_up, self.w_down = mk(experts, f, d), mk(experts, f, d), mk(experts, d, f)
        self.cos, self.sin = L.moe_rope_table(rope_frequencies(dim, **scaling).cuda(), n_pos)
        self.cache = PagedKVCache(pages, page_size, kv_heads, dim, eight_bit=eight_bit)
        self.attention = CachedAttention(self.cache, heads, self.w_qkv, self.w_out, self.cos, self.sin, axes=sections and rope_axes(sections))
        self._layers = {}

    def moe(self, x):
        """The MoE layer for this number of rows.  Its buffers are large (gradients of the weights among them), so that of the last two sizes are kept: a
        prompt's and a step's."""
        layer = self._layers.pop(len(x), None)
        while len(self._layers) > 1:
            del self._layers[next(iter(self._layers))]               # the one used longest ago, before another is made
        if layer is None:
            layer = MoELayer(len(x), self.d, self.experts, self.k, self.f, torch.bfloat16, self.w_gate, self.w_up, self.w_down, w_router=self.w_router, gather=True,
                             save_gu=False)
        self._layers[len(x)] = layer
        return layer.forward(x)

    @staticmethod
    def norm(x):
        return L.moe_norm_fwd(x, eps=1e-6, rms=True, stats=False)[0]

    def _rest(self, x, y):
        normed, x, _, _ = L.moe_norm_fwd(y, eps=1e-6, rms=True, residual=x, stats=False)
        return x + self.moe(normed)

    def prompt(self, x, seqs, counts, positions=None):
        return self._rest(x, self.attention.prompt(self.norm(x), seqs, counts, positions))

    def token(self, x, seqs):
        return self._rest(x, self.attention.token(self.norm(x), seqs))


def picture_then_text(count, rows, cols):
    """Positions [3, count] of a picture of rows x cols patches (fewer, if the prompt ends before) and the text after it."""
    patch = torch.arange(min(count, rows * cols))
    picture = torch.stack((torch.zeros_like(patch), patch // cols, patch % cols))
    text = torch.arange(max(rows, cols), max(rows, cols) + count - len(patch)).expand(3, -1)
    return torch.cat((picture, text), dim=1).int()


def generate(block, prompts, tokens, positions=None):
    """prompts: [n_i, d] bf16 per sequence, positions [axes, sum n_i] of theirs if they are not text alone -> the rows that every sequence went through,
    [tokens + 1, sequences, d]."""
    seqs, counts = list(range(len(prompts))), [len(p) for p in prompts]
    for s in seqs:
        block.cache.open(s)
    y = block.prompt(torch.cat(prompts), seqs, counts, positions)
    ends = torch.tensor(counts).cumsum(0) - 1
    rows = [y[ends.to(y.device)]]
    for _ in range(tokens):
        rows.append(block.token(rows[-1], seqs))
    for s in seqs:
        block.cache.close(s)
    return torch.stack(rows)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--seqs", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=300, help="tokens of the longest prompt")
    ap.add_argument("--tokens", type=int, default=32)
    ap.add_argument("--bf16-cache", action="store_true")
    ap.add_argument("--pictures", action="store_true", help="every prompt begins with a picture of 8 x 8 patches; positions have three axes")
    a = ap.parse_args()
    lens = [max(1, a.prompt * (i + 1) // a.seqs) for i in range(a.seqs)]
    n_pos = a.prompt + a.tokens
    block = Block(2048, 32, 4, 128, 128, 8, 768, pages=sum(-(-(n + a.tokens) // 16) for n in lens), page_size=16, n_pos=n_pos, eight_bit=not a.bf16_cache, base=1e6,
                  sections=(16, 24, 24) if a.pictures else None)
    positions = torch.cat([picture_then_text(n, 8, 8) for n in lens], dim=1) if a.pictures else None
    prompts = [torch.randn((n, 2048), device="cuda").bfloat16() for n in lens]
    generate(block, prompts, 2, positions)
    torch.cuda.synchronize()
    began = time.perf_counter()
    rows = generate(block, prompts, a.tokens, positions)
    torch.cuda.synchronize()
    s = time.perf_counter() - began
    print("%d sequences, %d prompt tokens, %d steps: %.1f ms in all, last rows' rms %.3f" % (a.seqs, sum(lens), a.tokens, 1e3 * s, rows[-1].float().square().mean().sqrt().item()))


if __name__ == "__main__":
    main()
