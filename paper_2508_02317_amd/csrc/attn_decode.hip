// Attention of one new token per sequence over a paged key/value cache, split over the contexts' length and joined.
//
//     out[b, h] = sum_t p_t v_t / sum_t p_t,   p_t = exp(scale <q[b, h], k_t> - m),   m = max_t scale <q[b, h], k_t>
//
// All heads of a group share their keys and values, so an element of the cache is read once and used for the whole group: 16 operations
// per byte at most (bf16, 16 heads; 31 in 8 bits), far below what the matrix units need to be busy.  The kernel is bound by the rate at which the cache
// arrives, and its layout serves that rate:
//
//   * No key or value passes through LDS.  A wave takes kSub tokens at a time, and the operands of the matrix instructions are what its lanes
//     load, 16 bytes each.  With lane = 16 c + n:
//       scores   S^T = K Q^T   row = token 16 a + n of the wave's tokens (a = 0, 1), column = head n, reduction along the head's elements
//                              in any order that keys and queries share: a lane reads 16 bytes of its token's row
//       result   lane holds the scores of head n and the tokens 16 a + 4 c + r (r = 0..3)
//       output   O^T = V^T P^T row = element, column = head n, reduction along tokens, in any order that values and p share: the order in
//                              which the scores lie already, so p goes from one product to the next without leaving its lane.  A
//                              lane reads the elements [n * kE, + kE) of the tokens 16 a + 4 c + r, whole rows of memory per 16 lanes, and one byte
//                              permutation per pair of tokens makes the operand
//     A head's scores, maximum, sum and output elements are all in the lanes of the same n: the running rescaling is lane-local.
//   * The loads of the next tokens are in flight while these are worked on: keys from the moment the scores are formed, values from the moment
//     the output is.  Every byte offset of a lane is the same for all tokens; pages enter as scalar bases, their ids read a round ahead.
//     Values are streamed past the caches, keys are not: a lane reads 64-byte pieces of key rows, so that the second half of a line comes
//     from the cache (64 contexts of 8192 tokens, 4 key heads of 128 elements in bf16: 173 us; values kept 193; keys streamed 174, but
//     16 contexts of 4096, which the last-level cache holds from one call to the next, 27 -> 30 us).
//   * The tokens of all sequences and heads form one line of tiles of 4 kSub tokens, cut into equal pieces, one per workgroup: lengths may
//     differ as they like.  A workgroup that does not see the whole context of a head leaves its maximum, sum and unscaled output behind, at most
//     two of them, and a second launch joins those.  The cut depends on lens alone, so results do not change from call to call.  Tiles of kSub tokens
//     would cut more evenly but leave three waves of four idle in a workgroup's last round: 16 contexts of up to 4096 tokens 24 -> 29.5 us.
//     512 workgroups (256 for heads of more than 128 elements) are what the card has room for; 768 and 1024 were 2 to 8 % slower.
//     Eight waves on half as many workgroups: 64 contexts of 8192 tokens 1 to 3 % faster, one of 100 to 1000 15 to 20 % slower.
//
// Scores are fp32 sums of exact products (8-bit values are exact in bf16).  p is split into two bf16 numbers, together exact to 2^-16, so that
// rounding it leaves the result as if it had not been rounded; one alone made the error against 64 bits 1.01 to 1.04 times as large, and the second
// product takes nothing in bf16 and up to 2 % with an 8-bit cache.
//
// Measured on one MI355X, both launches: 128 contexts of 8192 tokens (4 key heads of 128 elements, 32 query heads, bf16, 2.1 GB) 320 us, 6.8 TB/s
// in the first launch, where a kernel that reads and does nothing else has 7.0; 64 contexts of up to 8192, 548 MB, 94 to 97 us; 32 of up to
// 40960 in 8 bits, 702 MB, 119 to 124 us (5.9 TB/s: the vector unit is busy four tenths of the time, the matrix unit an eighth).  What is missing on shorter
// calls is fixed: about 5 us from the launch to the first keys (arguments, lengths, page ids and keys, each waited for by the next), 3 at the
// end and 3 to 5 for the join.
#include <cmath>
#include <type_traits>
#include "attn_plan.h"
#include "launch_plan.h"
#include "moe_common.h"
#include "mx8_codes.h"

namespace moe {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x1 __attribute__((ext_vector_type(1)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int kJoinAhead = 4;                          // pieces that a lane of the join has in flight
constexpr double kLog2e = 1.44269504088896340736;
constexpr float kLn2 = 0.69314718055994530942f;

struct Args {
  const void* q;
  int64_t q_stride_b, q_stride_h;
  const char *k, *v, *ks, *vs;
  int64_t page_bytes, scale_page_bytes;               // from one page to the next
  int pages, page_shift;
  const int32_t *block_table, *lens;
  int max_pages, B, Hq, Hkv, group, parts, heads;      // group: query heads per key head, in `parts` units of up to `heads`
  float scale_hi, scale_lo;                            // together scale log2 e
  int window, tile_subs;                              // tile_subs: stretches of kSub tokens in a tile, four of them or a whole context
  void* out;
  float* lse;
  int32_t* unit_pieces;                                // [B * Hkv * parts][2]: first workgroup (its slot in bit 0) and last of a cut unit, or -1
  float* slots;                                        // [2 W][heads][D + 4]: maximum, sum, two unused, output
};

__device__ __forceinline__ float row_max4(float v) {   // over the four lanes of the same n
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum4(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// 16 rows of a page as a buffer: a lane's offset is the same for all tokens, and rows that are not there (range 0) are not fetched, so that loads
// ahead need no branch around them.
struct Rows {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ Rows(const char* first, uint32_t range) {
    rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(first), 0, static_cast<int>(range), 0x00020000);
  }
  // aux 2: streamed
  template <class V, int AUX> __device__ __forceinline__ V load(uint32_t off) const {
    if constexpr (sizeof(V) == 16) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(rsrc, static_cast<int>(off), 0, AUX));
    else if constexpr (sizeof(V) == 8) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b64(rsrc, static_cast<int>(off), 0, AUX));
    else if constexpr (sizeof(V) == 4) return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b32(rsrc, static_cast<int>(off), 0, AUX));
    else return __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b16(rsrc, static_cast<int>(off), 0, AUX));
  }
};
// N consecutive words in the widest vectors that divide them.
template <int N> struct Words {
  typedef std::conditional_t<N % 4 == 0, u32x4, std::conditional_t<N % 2 == 0, u32x2, u32x1>> V;
  static constexpr int kLanes = sizeof(V) / 4;
  V w[N / kLanes];
  template <int AUX> __device__ __forceinline__ void load(const Rows& rows, uint32_t off) {
#pragma unroll
    for (int i = 0; i < N / kLanes; ++i) w[i] = rows.template load<V, AUX>(off + i * static_cast<int>(sizeof(V)));
  }
  __device__ __forceinline__ uint32_t operator[](int i) const { return w[i / kLanes][i % kLanes]; }
  __device__ __forceinline__ void put(int i, uint32_t x) { w[i / kLanes][i % kLanes] = x; }
};

// N bytes that begin at a multiple of N: whole words where N is one, else pairs of bytes.
template <int N> struct ScaleRow {
  typedef std::conditional_t<N % 4 == 0, Words<(N + 3) / 4>, uint16_t[(N + 1) / 2]> V;
  V v;
  __device__ __forceinline__ void load(const Rows& rows, uint32_t off) {
    if constexpr (N % 4 == 0) {
      v.template load<0>(rows, off);
    } else {
#pragma unroll
      for (int i = 0; i < N / 2; ++i) v[i] = rows.template load<uint16_t, 0>(off + 2 * i);
    }
  }
  __device__ __forceinline__ uint32_t pair(int i) const {   // bytes 2 i and 2 i + 1
    if constexpr (N % 4 == 0) return v[i / 2] >> (16 * (i % 2));
    else return v[i];
  }
};

// What a wave holds of its tokens, and the products with it.
template <int KIND, int D> struct Wave {
  static constexpr bool kF32 = KIND == MOE_F32, kMx = KIND == MOE_MX8;
  static constexpr int kHalves = attn_halves(KIND, D), kSub = 16 * kHalves, kStep = kWaves * kSub;   // tokens of a wave, of a workgroup at a time
  static constexpr int kG = !kF32 && D % 128 == 0 ? 128 : 64, kE = kG / 16, kNG = D / kG;   // a lane's values: kE elements of each of kNG groups of kG
  static constexpr int kEs = kF32 ? 4 : kMx ? 1 : 2, kRow = D * kEs;               // bytes of an element, of a token's row
  static constexpr int kKPieces = kMx ? D / 64 : kF32 ? D / 16 : D / 32;           // 16-byte pieces of a key row that a lane reads
  static constexpr int kKStep = 64;                                                // bytes between them (4 lanes of 16 bytes)
  static constexpr int kVTokens = 4 * kHalves, kVWords = kE * kEs / 4;             // tokens and words of a group that a lane reads of the values
  static constexpr int kScaleRow = D / 32;                                         // scale bytes of a token
  static constexpr int kQPieces = kF32 ? D / 16 : D / 32;                          // 16-byte pieces of a query that a lane holds

  u32x4 k[kHalves][kKPieces];
  Words<kVWords> v[kVTokens][kNG];
  ScaleRow<kMx ? kScaleRow : 4> ks[kMx ? kHalves : 1];  // a token's scale bytes
  Words<kMx ? kScaleRow : 1> vs[kMx ? kHalves : 1];      // 4 tokens' scale bytes
  u32x4 q[kQPieces], q_next[kQPieces];                   // of this part of the piece and of the next
  f32x4 acc[kNG][kE];
  float m, l;

  __device__ __forceinline__ void load_q(const char* head_row, int c) {
#pragma unroll
    for (int i = 0; i < kQPieces; ++i) {
      // the elements that the keys' lane holds: bytes 64 i + 16 c on, or for 8-bit keys the elements 64 (i / 2) + 16 c + 8 (i % 2) on
      const int at = kMx ? ((i / 2) * 64 + c * 16 + (i % 2) * 8) * 2 : i * 64 + c * 16;
      q_next[i] = *reinterpret_cast<const u32x4*>(head_row + at);
    }
  }
  __device__ __forceinline__ void take_q() {
#pragma unroll
    for (int i = 0; i < kQPieces; ++i) q[i] = q_next[i];
  }
  __device__ __forceinline__ void begin() {
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int g = 0; g < kNG; ++g)
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[g][e] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // half a's 16 tokens: their rows and the rows of their scales; n, c: of the lane
  __device__ __forceinline__ void load_k(int a, const Rows& rows, const Rows& scales, int n, int c) {
#pragma unroll
    for (int i = 0; i < kKPieces; ++i) k[a][i] = rows.template load<u32x4, 0>(n * kRow + c * 16 + i * kKStep);
    if constexpr (kMx) ks[a].load(scales, n * kScaleRow);
  }
  __device__ __forceinline__ void load_v(int a, const Rows& rows, const Rows& scales, int n, int c) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int g = 0; g < kNG; ++g) v[4 * a + r][g].template load<2>(rows, c * 4 * kRow + n * kE * kEs + r * kRow + g * kG * kEs);
    if constexpr (kMx) vs[a].template load<0>(scales, c * 4 * kScaleRow);
  }
  // eight codes (two words) -> eight bf16
  static __device__ __forceinline__ bf16x8 decode8(uint32_t w0, uint32_t w1, float s) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, s, true);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, false), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, s, true);
    return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
  }
  // In fp32, four products of one chain of additions after the other: two chains are half as long, in time and in rounding.
  static constexpr int kChains = kF32 ? 2 : 1;
  __device__ __forceinline__ void scores(f32x4 (&s)[kHalves], int c) const {
    f32x4 t[kHalves][kChains];
#pragma unroll
    for (int a = 0; a < kHalves; ++a)
#pragma unroll
      for (int u = 0; u < kChains; ++u) t[a][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kKPieces; ++i)
#pragma unroll
      for (int a = 0; a < kHalves; ++a) {
        if constexpr (kF32) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            t[a][j % kChains] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[a][i][j]), __uint_as_float(q[i][j]), t[a][j % kChains], 0, 0, 0);
        } else if constexpr (kMx) {
          const float sc = mx_scale((ks[a].pair(i) >> (8 * (c >> 1))) & 0xFFu);
#pragma unroll
          for (int h = 0; h < 2; ++h)
            t[a][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(k[a][i][2 * h], k[a][i][2 * h + 1], sc), __builtin_bit_cast(bf16x8, q[2 * i + h]), t[a][0], 0, 0, 0);
        } else {
          t[a][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[a][i]), __builtin_bit_cast(bf16x8, q[i]), t[a][0], 0, 0, 0);
        }
      }
#pragma unroll
    for (int a = 0; a < kHalves; ++a) {
      s[a] = t[a][0];
#pragma unroll
      for (int u = 1; u < kChains; ++u) s[a] += t[a][u];
    }
  }
  // p of the scores, with the running maximum, sum and output brought to the new maximum.  Exponents are of 2: x = s (hi + lo) with
  // hi + lo = scale log2 e.  The maximum is one of the rounded products s hi; an exponent is formed from s anew, so that it has
  // the rounding of a small difference and not that of the product.  `mask`: bit 4 a + r set where this lane's token exists.
  __device__ __forceinline__ void softmax(f32x4 (&s)[kHalves], float hi, float lo, uint32_t mask) {
    f32x4 x[kHalves];
    float top = -INFINITY;
#pragma unroll
    for (int a = 0; a < kHalves; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[a][r] = (mask >> (4 * a + r)) & 1u ? s[a][r] * hi : -INFINITY;
        top = fmaxf(top, x[a][r]);
      }
    top = fmaxf(m, row_max4(top));
    if (__any(top > m)) {
      const float f = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.0f;   // m = -inf: 0
      l *= f;
#pragma unroll
      for (int g = 0; g < kNG; ++g)
#pragma unroll
        for (int e = 0; e < kE; ++e) acc[g][e] *= f;
      m = top;
    }
    const float base = m > -INFINITY ? m : 0.0f;
#pragma unroll
    for (int a = 0; a < kHalves; ++a)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[a][r], lo, fmaf(s[a][r], hi, -base)));
        s[a][r] = x[a][r] == -INFINITY ? 0.0f : p;     // masked, or a score of -inf: no weight (and a NaN stays one)
        l += s[a][r];
      }
  }
  // Values of tokens that do not exist become zeros: their p is 0, but what lies there may be infinite or NaN.
  __device__ __forceinline__ void clear_missing(uint32_t mask) {
#pragma unroll
    for (int t = 0; t < kVTokens; ++t) {
      const bool there = (mask >> t) & 1u;
#pragma unroll
      for (int g = 0; g < kNG; ++g)
#pragma unroll
        for (int i = 0; i < kVWords; ++i) v[t][g].put(i, there ? v[t][g][i] : 0u);
      if constexpr (kMx) {                             // and the scales: a scale code of 255 stands for NaN
#pragma unroll
        for (int i = 0; i < kScaleRow; ++i) {          // word i of the four tokens' bytes
          uint32_t bytes = 0u;
#pragma unroll
          for (int b = 0; b < 4; ++b) bytes |= (4 * i + b) / kScaleRow == t % 4 ? 0xFFu << (8 * b) : 0u;
          if (bytes != 0u) vs[t / 4].put(i, there ? vs[t / 4][i] : vs[t / 4][i] & ~bytes);
        }
      }
    }
  }
  // out += values * p
  __device__ __forceinline__ void output(const f32x4 (&p)[kHalves], int n) {
    if constexpr (kF32) {
#pragma unroll
      for (int r = 0; r < kVTokens; ++r)
#pragma unroll
        for (int g = 0; g < kNG; ++g)
#pragma unroll
          for (int e = 0; e < kE; ++e)
            acc[g][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[r][g][e]), p[r / 4][r % 4], acc[g][e], 0, 0, 0);
    } else {
#pragma unroll
     for (int two = 0; two < kHalves; two += 2) {
      u32x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {                    // tokens 16 (two + i / 2) + 4 c + 2 (i % 2) and the next
        const float x = p[two + i / 2][2 * (i % 2)], y = p[two + i / 2][2 * (i % 2) + 1];
        hi[i] = pack_bf16x2(x, y);
        lo[i] = pack_bf16x2(x - bf16_lo(hi[i]), y - bf16_hi(hi[i]));
      }
      const bf16x8 ph = __builtin_bit_cast(bf16x8, hi), pl = __builtin_bit_cast(bf16x8, lo);
#pragma unroll
      for (int g = 0; g < kNG; ++g) {
        uint32_t w[8][kE / 2];                         // bf16 pairs of the lane's elements, by token
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const int vt = 4 * two + t;
          if constexpr (kMx) {
            const int at = (t & 3) * kScaleRow + g * (kG / 32);        // byte of the first of the row's scales for this group
            const float sc = mx_scale((vs[vt >> 2][at >> 2] >> (8 * ((at & 3) + n * kE / 32))) & 0xFFu);
#pragma unroll
            for (int e = 0; e < kE / 4; ++e) {
              w[t][2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[vt][g][e], sc, false));
              w[t][2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[vt][g][e], sc, true));
            }
          } else {
#pragma unroll
            for (int e = 0; e < kE / 2; ++e) w[t][e] = v[vt][g][e];
          }
        }
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          u32x4 x;
#pragma unroll
          for (int i = 0; i < 4; ++i)                  // element e of two tokens
            x[i] = __builtin_amdgcn_perm(w[2 * i + 1][e / 2], w[2 * i][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
          acc[g][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), ph, acc[g][e], 0, 0, 0);
          acc[g][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), pl, acc[g][e], 0, 0, 0);
        }
      }
     }
    }
  }
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

template <int KIND, int D>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2) void attn_decode_kernel(Args a) {
  typedef Wave<KIND, D> W;
  typedef std::conditional_t<KIND == MOE_F32, float, bf16_t> E;
  constexpr int kPad = D + 4;
  __shared__ float s_out[kWaves][16][kPad];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];
  const int lane = static_cast<int>(threadIdx.x) & 63, wave = uniform(static_cast<int>(threadIdx.x) >> 6), n = lane & 15, c = lane >> 4;
  const int units = a.Hkv * a.parts, me = static_cast<int>(blockIdx.x);
  const int held = a.max_pages << a.page_shift;

  // Tiles of all sequences, and the sequence in which this workgroup's piece begins.  Every wave finds them for itself, four consecutive
  // sequences a lane, without a barrier: a load, a scan over the lanes, a ballot.
  const ScalarInts lens = scalar_ints(a.lens);
  // (a whole context is one tile of any length: with constants there is no division)
  auto span_of = [&](int len) { return a.unit_pieces ? attn_span(len, held, a.window, W::kSub, W::kStep) : attn_span(len, held, a.window, W::kSub, 1 << 30); };
  int len4[4], nt[4], mine = 0, incl = 0;              // of this lane's sequences: lengths, tiles of each, their sum, the sum up to and with this lane
  bool empty = false;                                  // some sequence has no tokens
  auto count_from = [&](int b0) {
    mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int b = b0 + 4 * lane + j;
      len4[j] = b < a.B ? a.lens[b] : 0;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      nt[j] = span_of(len4[j]).tiles;
      mine += nt[j];
      empty |= nt[j] == 0 && b0 + 4 * lane + j < a.B;
    }
    incl = wave_inclusive_sum(mine);
    return __builtin_amdgcn_readlane(incl, 63);
  };
  int total = 0;
  for (int b0 = 0; b0 < a.B; b0 += 256) total += count_from(b0);
  const AttnCut cut = attn_cut(total * units, static_cast<int>(gridDim.x));
  const int at = attn_begin(cut, me);
  const int end = attn_begin(cut, me + 1);
  int b_at = 0, before = 0, len_at = 0;                // sequence of tile `at`, tiles (of one unit) of the sequences before it, its length
  if (at < end) {
    for (int b0 = 0;; b0 += 256) {
      const int here = a.B > 256 ? count_from(b0) : total;
      if (at >= (before + here) * units) { before += here; continue; }
      const int l = __builtin_ctzll(__ballot((before + incl) * units > at));   // the first lane whose sequences end behind the tile
      before += __builtin_amdgcn_readlane(incl - mine, l);
      b_at = b0 + 4 * l;
      len_at = __builtin_amdgcn_readlane(len4[0], l);
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        const int n_j = __builtin_amdgcn_readlane(nt[j], l);
        if (b_at == b0 + 4 * l + j && at >= (before + n_j) * units) {
          before += n_j;
          ++b_at;
          len_at = __builtin_amdgcn_readlane(len4[j + 1], l);
        }
      }
      break;
    }
  }

  for (int b = __any(empty) ? me : a.B; b < a.B; b += static_cast<int>(gridDim.x)) {
    if (span_of(lens[b]).tiles != 0) continue;
    for (int i = threadIdx.x; i < a.Hq * D; i += kThreads) static_cast<E*>(a.out)[static_cast<int64_t>(b) * a.Hq * D + i] = 0;
    if (a.lse)
      for (int i = threadIdx.x; i < a.Hq; i += kThreads) a.lse[static_cast<int64_t>(b) * a.Hq + i] = -INFINITY;
    if (a.unit_pieces)
      for (int i = threadIdx.x; i < units; i += kThreads) a.unit_pieces[2 * (static_cast<int64_t>(b) * units + i)] = -1;
  }

  // A stretch of the piece within one unit (a sequence and a group of heads), and what of it is this wave's: every fourth of its stretches of
  // kSub tokens, `rounds` of them from token t0 on; nothing is fetched from `until` on.
  struct Part {
    int b, head0, heads, kv, unit_begin, unit_end, first, last, lo, len, t0, rounds, until, u;
    ScalarInts pages;
  };
  auto part_at = [&](int tile) {
    AttnSpan sp = span_of(len_at);
    while (tile >= (before + sp.tiles) * units) {      // on to the sequence that has the tile
      before += sp.tiles;
      len_at = lens[++b_at];
      sp = span_of(len_at);
    }
    Part q;
    q.b = b_at;
    q.u = quotient(tile - before * units, sp.tiles);
    q.unit_begin = before * units + q.u * sp.tiles;
    q.unit_end = q.unit_begin + sp.tiles;
    q.first = tile;
    q.last = min(end, q.unit_end);
    q.kv = a.parts == 1 ? q.u : quotient(q.u, a.parts);
    const int part = q.u - q.kv * a.parts;
    q.head0 = q.kv * a.group + part * a.heads;
    q.heads = min(a.heads, a.group - part * a.heads);
    q.lo = sp.lo;
    q.len = sp.len;
    const int sub0 = (tile - q.unit_begin) * a.tile_subs + wave, sub1 = min((q.last - q.unit_begin) * a.tile_subs, quotient(sp.len - sp.base + W::kSub - 1, W::kSub));
    q.t0 = sp.base + sub0 * W::kSub;
    q.rounds = sub0 < sub1 ? quotient(sub1 - sub0 + kWaves - 1, kWaves) : 0;
    q.until = sub0 < sub1 ? min(sp.len, sp.base + sub1 * W::kSub) : 0;
    q.pages = scalar_ints(a.block_table + static_cast<int64_t>(b_at) * a.max_pages);
    return q;
  };
  const int page_mask = (1 << a.page_shift) - 1;
  // A half of 16 tokens that begins at token t lies in one page.  A half without tokens takes the nearest one that has some, and is masked.
  auto near = [&](const Part& q, int t) { return min(max(t, q.lo), q.len - 1); };
  W w;
  int page[W::kHalves];                                // of the tokens whose loads are issued next, requested one round ahead
  int64_t row[W::kHalves], scale[W::kHalves];
  auto find_pages = [&](const Part& q, int t) {
#pragma unroll
    for (int h = 0; h < W::kHalves; ++h) page[h] = q.pages[near(q, t + 16 * h) >> a.page_shift];
  };
  auto load_k = [&](const Part& q, int t) {            // into the pages that were found, whose rows the values' loads use too
#pragma unroll
    for (int h = 0; h < W::kHalves; ++h) {
      const int in_page = (q.kv << a.page_shift) + (near(q, t + 16 * h) & page_mask & ~15);
      const int64_t p = min(max(page[h], 0), a.pages - 1);
      row[h] = p * a.page_bytes + static_cast<int64_t>(in_page) * W::kRow;
      scale[h] = p * a.scale_page_bytes + static_cast<int64_t>(in_page) * W::kScaleRow;
    }
#pragma unroll
    for (int h = 0; h < W::kHalves; ++h) {
      const bool there = t + 16 * h < q.until;
      w.load_k(h, Rows(a.k + row[h], there ? 16 * W::kRow : 0), Rows(a.ks + scale[h], there ? 16 * W::kScaleRow : 0), n, c);
    }
  };
  auto load_v = [&](const Part& q, int t) {
#pragma unroll
    for (int h = 0; h < W::kHalves; ++h) {
      const bool there = t + 16 * h < q.until;
      w.load_v(h, Rows(a.v + row[h], there ? 16 * W::kRow : 0), Rows(a.vs + scale[h], there ? 16 * W::kScaleRow : 0), n, c);
    }
  };
  auto load_q = [&](const Part& q) {
    const int h = q.head0 + min(n, q.heads - 1);       // columns without a head repeat the last one's
    w.load_q(static_cast<const char*>(a.q) + (static_cast<int64_t>(q.b) * a.q_stride_b + static_cast<int64_t>(h) * a.q_stride_h) * static_cast<int>(sizeof(E)), c);
  };
  if (at >= end) return;
  Part cur = part_at(at);
  load_q(cur);
  find_pages(cur, cur.t0);
  load_k(cur, cur.t0);
  __builtin_amdgcn_sched_barrier(0);                   // the order of the rounds: keys are the older ones when scores wait for them
  load_v(cur, cur.t0);

  for (;;) {
    // what comes after this part; behind the piece's end: this part again, with nothing to fetch
    Part next = cur;
    next.until = next.rounds = 0;
    if (cur.last < end) next = part_at(cur.last);
    const int lo = cur.lo, len = cur.len, heads = cur.heads;
    w.take_q();
    if (cur.last < end) load_q(next);
    w.begin();
    int t0 = cur.t0;
    if (cur.rounds > 1) find_pages(cur, t0 + W::kStep); else find_pages(next, next.t0);
    // The next keys are requested as soon as the scores are formed, the next values after the output, the first ones of the next part among
    // them, and where nothing follows with a range of nothing: without branches around the requests a wait for older ones leaves the younger
    // ones in flight.
    for (int i = 1; i <= cur.rounds; ++i) {
      f32x4 s[W::kHalves];
      w.scores(s, c);
      const Part& from = i < cur.rounds ? cur : next;
      const int t1 = i < cur.rounds ? t0 + W::kStep : next.t0;
      load_k(from, t1);
      if (i + 1 < cur.rounds) find_pages(cur, t1 + W::kStep); else find_pages(next, next.t0);
      const bool whole = t0 >= lo && t0 + W::kSub <= len;
      uint32_t mask = ~0u;
      if (!whole) {
        mask = 0u;
#pragma unroll
        for (int h = 0; h < W::kHalves; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int t = t0 + 16 * h + 4 * c + r;
            mask |= t >= lo && t < len ? 1u << (4 * h + r) : 0u;
          }
      }
      w.softmax(s, a.scale_hi, a.scale_lo, mask);
      if (!whole) w.clear_missing(mask);
      w.output(s, n);
      load_v(from, t1);
      t0 = t1;
    }
    if (cur.rounds == 0) {                             // nothing of this part was this wave's, so nothing has been requested behind it
      load_k(next, next.t0);
      load_v(next, next.t0);
    }

    // the four waves' parts, each to its own maximum, and out
    const float l = row_sum4(w.l);
    if (lane < 16) { s_m[wave][n] = w.m; s_l[wave][n] = l; }
    if (n < heads) {
#pragma unroll
      for (int g = 0; g < W::kNG; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int e = 0; e < W::kE; e += 4)
            *reinterpret_cast<f32x4*>(&s_out[wave][n][g * W::kG + (4 * c + r) * W::kE + e]) = f32x4{w.acc[g][e][r], w.acc[g][e + 1][r], w.acc[g][e + 2][r], w.acc[g][e + 3][r]};
    }
    __syncthreads();
    const bool complete = cur.first == cur.unit_begin && cur.last == cur.unit_end;
    const int slot = 2 * me + (cur.first == at ? 0 : 1);
    for (int i = threadIdx.x; i < heads * (D / 4); i += kThreads) {
      const int h = i / (D / 4), d = (i - h * (D / 4)) * 4;
      const float m = fmaxf(fmaxf(s_m[0][h], s_m[1][h]), fmaxf(s_m[2][h], s_m[3][h]));
      float sum = 0.0f;
      f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float f = s_m[v][h] > -INFINITY ? __builtin_amdgcn_exp2f(s_m[v][h] - m) : 0.0f;
        sum += s_l[v][h] * f;
        o += *reinterpret_cast<const f32x4*>(&s_out[v][h][d]) * f;
      }
      if (complete) {
        const int64_t row = static_cast<int64_t>(cur.b) * a.Hq + cur.head0 + h;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        if constexpr (KIND == MOE_F32) {
          *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + row * D + d) = o * inv;
        } else {
          *reinterpret_cast<u32x2*>(static_cast<bf16_t*>(a.out) + row * D + d) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
        }
        if (a.lse && d == 0) a.lse[row] = (m + log2f(sum)) * kLn2;
      } else {
        float* to = a.slots + (static_cast<int64_t>(slot) * a.heads + h) * (D + 4);
        *reinterpret_cast<f32x4*>(to + 4 + d) = o;
        if (d == 0) { to[0] = m; to[1] = sum; }
      }
    }
    if (a.unit_pieces && threadIdx.x == 0 && cur.first == cur.unit_begin) {
      int32_t* p = a.unit_pieces + 2 * (static_cast<int64_t>(cur.b) * units + cur.u);
      p[0] = complete ? -1 : slot;
      p[1] = attn_owner(cut, cur.unit_end - 1);
    }
    if (cur.last >= end) return;
    __syncthreads();                                   // the sums have been read
    cur = next;
  }
}

// ---- pieces of a context joined: a workgroup per sequence and head ---------------------------------------
// A slice of lanes takes every kSlices-th piece, maximum, sum and output at once and kAhead pieces in flight; the slices meet in LDS.
template <int KIND, int D, int THREADS>
__global__ __launch_bounds__(THREADS) void attn_join_kernel(Args a) {
  typedef std::conditional_t<KIND == MOE_F32, float, bf16_t> E;
  constexpr int kCols = D / 4, kSlices = THREADS / kCols, kAhead = kJoinAhead;
  __shared__ float s_m[kSlices], s_l[kSlices];
  __shared__ float s_out[kSlices][D];
  const int units = a.Hkv * a.parts, tid = static_cast<int>(threadIdx.x);
  const int b = blockIdx.x / a.Hq, head = blockIdx.x - b * a.Hq, kv = head / a.group, in_group = head - kv * a.group;
  const int part = in_group / a.heads, h = in_group - part * a.heads;
  const ScalarInts p = scalar_ints(a.unit_pieces + 2 * (static_cast<int64_t>(b) * units + kv * a.parts + part));
  const int slot0 = p[0], w0 = slot0 >> 1, count = p[1] - w0 + 1;
  if (slot0 < 0) return;
  const int slice = tid / kCols, d = (tid - slice * kCols) * 4;
  if (slice < kSlices) {
    float m = -INFINITY, l = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = slice; i0 < count; i0 += kAhead * kSlices) {
      float mi[kAhead], li[kAhead];
      f32x4 oi[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = min(i0 + j * kSlices, count - 1);
        // the first piece may be its workgroup's second; all others are their workgroup's first
        const float* at = a.slots + (static_cast<int64_t>(i == 0 ? slot0 : 2 * (w0 + i)) * a.heads + h) * (D + 4);
        mi[j] = at[0];
        li[j] = at[1];
        oi[j] = *reinterpret_cast<const f32x4*>(at + 4 + d);
      }
      float top = m;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) top = i0 + j * kSlices < count ? fmaxf(top, mi[j]) : top;
      const float base = top > -INFINITY ? top : 0.0f;   // a maximum of -inf counts with weight 0
      const float f = __builtin_amdgcn_exp2f(m - base);
      l *= f;
      o *= f;
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const float g = i0 + j * kSlices < count ? __builtin_amdgcn_exp2f(mi[j] - base) : 0.0f;
        l += li[j] * g;
        o += oi[j] * g;
      }
      m = top;
    }
    if (d == 0) { s_m[slice] = m; s_l[slice] = l; }
    *reinterpret_cast<f32x4*>(&s_out[slice][d]) = o;
  }
  __syncthreads();
  if (tid < kCols) {
    float top = s_m[0], sum = 0.0f;
#pragma unroll
    for (int s = 1; s < kSlices; ++s) top = fmaxf(top, s_m[s]);
    const float base = top > -INFINITY ? top : 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < kSlices; ++s) {
      const float f = __builtin_amdgcn_exp2f(s_m[s] - base);
      sum += s_l[s] * f;
      o += *reinterpret_cast<const f32x4*>(&s_out[s][d]) * f;
    }
    const int64_t row = static_cast<int64_t>(b) * a.Hq + head;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    if constexpr (KIND == MOE_F32) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + row * D + d) = o * inv;
    } else {
      *reinterpret_cast<u32x2*>(static_cast<bf16_t*>(a.out) + row * D + d) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
    }
    if (a.lse && d == 0) a.lse[row] = (top + log2f(sum)) * kLn2;
  }
}

// ---- host -------------------------------------------------------------------------------------------------
struct Launch { int sub, tile_subs, parts, heads, blocks; int64_t most_subs; bool cut; };
Launch launch_of(int dtype, int dim, int B, int Hq, int Hkv, int page_size, int max_pages, int window) {
  Launch l;
  l.sub = 16 * attn_halves(dtype, dim);
  const int group = Hq / Hkv;
  l.parts = ceil_div(group, 16);
  l.heads = ceil_div(group, l.parts);
  const int64_t units = static_cast<int64_t>(B) * Hkv * l.parts, held = static_cast<int64_t>(page_size) * max_pages;
  const int64_t most_seen = static_cast<int64_t>(window) + l.sub, seen = window > 0 && most_seen < held ? most_seen : held, subs = (seen + l.sub - 1) / l.sub;   // a window may begin inside a stretch
  // Contexts of few stretches are not cut (a context's one tile is the whole): a workgroup has it in a few turns, and no second launch is needed.  The
  // host does not have the lengths, so what the page table or the window has room for decides.
  // 4 key heads of 128 elements in bf16, cut -> whole: one context of 250 tokens 11.1 -> 7.9 us, 500 10.8 -> 9.5, 1000 10.8 -> 14.4; 64 contexts of
  // 250 14.4 -> 10.2, 500 18.4 -> 14.6, 1000 27.2 -> 23.6; 512 of 250 63 -> 54, 1000 180 -> 173.  All of equal lengths: whole contexts are dealt out by
  // their number, so ragged ones lose some of it (512 of up to 1000 tokens, 500 on average, 125 us; 512 of 500 95).
  l.cut = subs > (units >= 256 ? 32 : 16);
  l.tile_subs = l.cut ? kWaves : static_cast<int>(subs < 1 ? 1 : subs);
  l.most_subs = subs * units;
  const int64_t most = (l.cut ? (subs + kWaves - 1) / kWaves : 1) * units;
  const int at_once = dim > 128 ? kAttnMaxBlocks / 2 : kAttnMaxBlocks;   // as many as the card has room for: one or two a CU
  l.blocks = static_cast<int>(most < at_once ? most : at_once);
  if (l.blocks < 1) l.blocks = 1;
  return l;
}
// the larger of the element types' workspaces: the query does not know the cache's type
size_t pieces_bytes(int B, int Hkv, int parts) { return align_up(static_cast<size_t>(B) * Hkv * parts * 2 * sizeof(int32_t), 16); }
size_t ws_bytes_of(const Launch& l, int B, int Hkv, int dim) {
  return pieces_bytes(B, Hkv, l.parts) + static_cast<size_t>(l.blocks) * 2 * l.heads * (dim + 4) * sizeof(float);
}

template <int KIND, int D> void launch_decode(const Args& a, const Launch& l, hipStream_t st) {
  MOE_LAUNCH("attn_decode", (attn_decode_kernel<KIND, D>), dim3(l.blocks), dim3(kThreads), 0, st, a);
  if (!l.cut) return;
  // One wave per head where it has the pieces of a context in two goes, else four, which then need fewer goes.  one -> four, 4 key heads of 128
  // elements in bf16: 64 contexts of 8192 tokens (3 pieces each) 172.8 -> 173.2 us, of 64 elements 88.5 -> 89.4, with 16 heads to a key head 175.4 -> 177.1; one
  // context of 40960 (128) 28.6 -> 21.9.
  const dim3 joins(static_cast<unsigned>(a.B) * a.Hq);
  if (l.blocks <= static_cast<int64_t>(2 * kJoinAhead * (64 / (D / 4))) * a.B * a.Hkv * a.parts) MOE_LAUNCH("attn_join", (attn_join_kernel<KIND, D, 64>), joins, dim3(64), 0, st, a);
  else MOE_LAUNCH("attn_join", (attn_join_kernel<KIND, D, 256>), joins, dim3(256), 0, st, a);
}
template <int KIND> void launch_decode_dim(int dim, const Args& a, const Launch& l, hipStream_t st) {
  if (dim == 64) launch_decode<KIND, 64>(a, l, st);
  else if (dim == 128) launch_decode<KIND, 128>(a, l, st);
  else if (dim == 192) launch_decode<KIND, 192>(a, l, st);
  else launch_decode<KIND, 256>(a, l, st);
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_paged_attn_decode_workspace_bytes(int B, int Hq, int heads, int dim, int page_size, int max_pages) {
  if (B <= 0 || Hq <= 0 || heads <= 0 || dim <= 0 || page_size <= 0 || max_pages <= 0 || Hq % heads != 0) return 256;
  size_t most = 256;
  for (int dtype : {MOE_F32, MOE_BF16, MOE_MX8}) {
    const size_t need = ws_bytes_of(launch_of(dtype, dim, B, Hq, heads, page_size, max_pages, 0), B, heads, dim);
    if (need > most) most = need;
  }
  return most;
}

extern "C" int32_t moe_paged_attn_decode(const void* q, int64_t q_stride_b, int64_t q_stride_h, const moe_kv_cache_t* cache,
                                         const int32_t* block_table, int max_pages, const int32_t* lens, int B, int Hq, float scale,
                                         int window, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_cache("paged_attn_decode", cache)) return rc;
  MOE_REQUIRE(B >= 0 && Hq > 0 && max_pages >= 0 && window >= 0, MOE_ERR_INVALID_ARG, "paged_attn_decode: need B, max_pages, window >= 0 and Hq > 0 (B=%d Hq=%d max_pages=%d window=%d)",
              B, Hq, max_pages, window);
  MOE_REQUIRE(Hq % cache->heads == 0, MOE_ERR_INVALID_ARG, "paged_attn_decode: Hq=%d is no multiple of the cache's %d heads", Hq, cache->heads);
  MOE_REQUIRE(std::isfinite(scale), MOE_ERR_INVALID_ARG, "paged_attn_decode: scale is not finite");
  if (B == 0) return MOE_OK;
  const int el = cache->dtype == MOE_F32 ? 4 : 2;
  MOE_REQUIRE(q && lens && out && (max_pages == 0 || block_table), MOE_ERR_INVALID_ARG, "paged_attn_decode: null pointer");
  MOE_REQUIRE(aligned16(q) && aligned16(out) && aligned16(lse), MOE_ERR_INVALID_ARG, "paged_attn_decode: tensors must be 16-byte aligned");
  MOE_REQUIRE(q_stride_b % (16 / el) == 0 && q_stride_h % (16 / el) == 0, MOE_ERR_INVALID_ARG, "paged_attn_decode: strides must be multiples of 16 bytes");
  MOE_REQUIRE(static_cast<int64_t>(cache->page_size) * max_pages < (int64_t{1} << 31) - 4096, MOE_ERR_UNSUPPORTED, "paged_attn_decode: contexts of %lld tokens",
              static_cast<long long>(cache->page_size) * max_pages);
  MOE_REQUIRE(static_cast<int64_t>(B) * Hq <= (1 << 23), MOE_ERR_UNSUPPORTED, "paged_attn_decode: B * Hq = %lld above 2^23", static_cast<long long>(B) * Hq);
  const Launch l = launch_of(cache->dtype, cache->dim, B, Hq, cache->heads, cache->page_size, max_pages, window);
  MOE_REQUIRE(l.most_subs < (int64_t{1} << 31) - 65536, MOE_ERR_UNSUPPORTED, "paged_attn_decode: %lld stretches of %d tokens", static_cast<long long>(l.most_subs), l.sub);
  const size_t need = moe_paged_attn_decode_workspace_bytes(B, Hq, cache->heads, cache->dim, cache->page_size, max_pages);
  MOE_REQUIRE(ws && ws_bytes >= need && aligned16(ws), MOE_ERR_WORKSPACE, "paged_attn_decode: workspace null, misaligned or smaller than %zu bytes", need);
  Args a{};
  a.q = q; a.q_stride_b = q_stride_b; a.q_stride_h = q_stride_h;
  a.k = static_cast<const char*>(cache->k); a.v = static_cast<const char*>(cache->v);
  a.ks = static_cast<const char*>(cache->k_scales); a.vs = static_cast<const char*>(cache->v_scales);
  a.page_bytes = cache->page_stride * (cache->dtype == MOE_F32 ? 4 : cache->dtype == MOE_BF16 ? 2 : 1);
  a.scale_page_bytes = cache->scale_page_stride;
  a.pages = cache->pages; a.page_shift = __builtin_ctz(cache->page_size);
  a.block_table = block_table; a.lens = lens; a.max_pages = max_pages; a.B = B; a.Hq = Hq; a.Hkv = cache->heads; a.group = Hq / cache->heads;
  a.parts = l.parts; a.heads = l.heads; a.scale_hi = static_cast<float>(scale * kLog2e); a.scale_lo = static_cast<float>(scale * kLog2e - a.scale_hi); a.window = window; a.tile_subs = l.tile_subs; a.out = out; a.lse = lse;
  if (l.cut) {
    a.unit_pieces = static_cast<int32_t*>(ws);
    a.slots = reinterpret_cast<float*>(static_cast<char*>(ws) + pieces_bytes(B, cache->heads, l.parts));
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_paged_attn_decode", st);
  if (cache->dtype == MOE_F32) launch_decode_dim<MOE_F32>(cache->dim, a, l, st);
  else if (cache->dtype == MOE_BF16) launch_decode_dim<MOE_BF16>(cache->dim, a, l, st);
  else launch_decode_dim<MOE_MX8>(cache->dim, a, l, st);
  return end_call();
}
