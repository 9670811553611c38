// Which workgroup sees which tokens in the attention of one token over a paged cache: integer arithmetic without anything of a GPU in it,
// so that a plain C++ program can enumerate it (tests/test_attn_plan.py).
#pragma once
#include <stdint.h>

namespace moe {

constexpr int kAttnMaxBlocks = 512;                    // workgroups of a launch

// Stretches of 16 tokens that a wave has in registers at a time (kind as in moe.h: 0 fp32, 1 bf16, 2 8-bit blocks): two where a product reduces
// over 32 tokens, in fp32 as many as fit.  Twice as many in flight bought nothing: 64 contexts of 8192 tokens, 4 key heads, two -> four: bf16 of 64
// elements 90.0 -> 90.2 us, 8-bit of 64 54.5 -> 56.6, of 128 99.5 -> 104.
constexpr int attn_halves(int kind, int dim) { return kind == 0 && dim > 64 ? 1 : 2; }

// a / b of numbers that are not negative: without the signs' instructions
constexpr int quotient(int a, int b) { return static_cast<int>(static_cast<uint32_t>(a) / static_cast<uint32_t>(b)); }

// Tokens [lo, len) of a sequence are seen, in `tiles` tiles of `tile` tokens from `base` on, a multiple of `sub` at or below lo.
struct AttnSpan { int lo, len, base, tiles; };
constexpr AttnSpan attn_span(int len, int held, int window, int sub, int tile) {
  const int n = len < 0 ? 0 : len < held ? len : held;
  const int lo = window > 0 && n > window ? n - window : 0, base = quotient(lo, sub) * sub;
  return AttnSpan{lo, n, base, quotient(n - base + tile - 1, tile)};
}

// `total` tiles on `blocks` workgroups: the first `longer` of them take size + 1, the others size.
struct AttnCut { int size, longer; };
constexpr AttnCut attn_cut(int total, int blocks) {
  const int size = quotient(total, blocks);
  return AttnCut{size, total - size * blocks};
}
constexpr int attn_begin(const AttnCut& c, int block) { return block * c.size + (block < c.longer ? block : c.longer); }
// the workgroup that has a tile
constexpr int attn_owner(const AttnCut& c, int tile) {
  const int in_longer = c.longer * (c.size + 1);
  return tile < in_longer ? quotient(tile, c.size + 1) : c.longer + quotient(tile - in_longer, c.size > 0 ? c.size : 1);
}

}  // namespace moe
