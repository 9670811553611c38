// Rotary positions and the paged key/value cache: the rotation of queries and keys, forward and backward (RoPE is named among the
// efficient kernels, Sec. 3.2.5), the store of new keys and values into the cache's pages, in full or in 8 bits, and the way back.
//
// A pair of elements (a, b) of a head at position p is turned by the angle p w_i:
//     a' = a cos(p w_i) - b sin(p w_i),   b' = b cos(p w_i) + a sin(p w_i)
// with the pair (i, i + rot/2), or (2i, 2i + 1) where neighbours are paired; elements from rot on stay as they are.  The turn is a
// rotation, so its gradient is the turn by the opposite angle.
//
// Everything here moves bytes and is bound by HBM.  A lane owns 16 consecutive bytes of a head, so that a head row is contiguous over its
// lanes in every access; a row's lanes lie in one wave (up to 64 of them, rounded up to a power of two).  Tensors are streamed past the
// caches, table and scales are not.  Measured, in brackets with ordinary accesses: 40960 tokens of 32 + 4 heads of 128 elements in bf16, 755 MB,
// 124 us (142), 6.1 TB/s, the rate of a streaming copy; 8192 tokens 28 us (33), 5.4 TB/s; with keys and values stored into a cache 31 us (37),
// 5.5; 52949 cached tokens read back, 217 MB, 37 us (45), 5.8.  256 tokens of 16 heads take the 4 to 5 us of a launch.  8-bit rows: 33121 read back, 103 MB, 20 us, 5.2.
// The partner elements of the half layout come from the lane that owns them, not from memory again: a row is read whole before any
// of it is written, which makes the turn in place safe, and is read once.  The cosines and sines of a token are read once per lane and used for
// all heads that the lane walks.
// The products and the sum of a turn are rounded one by one (no fused multiply-add), as elementary operations in 32 bits round them: 8-bit
// codes are then the same decisions everywhere.
#include "launch_plan.h"
#include "moe_common.h"
#include "mx8_codes.h"

namespace moe {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kAtOnce = 4;                             // head rows whose loads a lane has in flight
constexpr int kBlocksWanted = 4096;                    // 8192 tokens of 36 heads: 29.1 us, 30.3 for 2048 and 29.6 for 8192; reads: 38.0, 38.7 for 1
constexpr int kMaxBlocksX = 1 << 20;                   // a workgroup walks on where there are more tokens

__device__ __forceinline__ int wave_of_block() { return __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6); }

// N consecutive elements of a head row as they lie in memory: 16 bytes, or 32 in fp32 rows of more than 64 pieces of 16.
template <class E, int N> struct Piece;
template <> struct Piece<bf16_t, 8> {
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)); }
  __device__ __forceinline__ void store(bf16_t* p) const { __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p)); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) { v[2 * q] = bf16_lo(w[q]); v[2 * q + 1] = bf16_hi(w[q]); }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = pack_bf16x2(v[2 * q], v[2 * q + 1]);
  }
  __device__ __forceinline__ Piece of_lane(int lane) const {
    Piece o;
#pragma unroll
    for (int q = 0; q < 4; ++q) o.w[q] = __shfl(w[q], lane, 64);
    return o;
  }
};
template <int N> struct Piece<float, N> {
  f32x4 w[N / 4];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int g = 0; g < N / 4; ++g) w[g] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p) + g);
  }
  __device__ __forceinline__ void store(float* p) const {
#pragma unroll
    for (int g = 0; g < N / 4; ++g) __builtin_nontemporal_store(w[g], reinterpret_cast<f32x4*>(p) + g);
  }
  __device__ __forceinline__ void get(float (&v)[N]) const {
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = w[q / 4][q % 4];
  }
  __device__ __forceinline__ void set(const float (&v)[N]) {
#pragma unroll
    for (int q = 0; q < N; ++q) w[q / 4][q % 4] = v[q];
  }
  __device__ __forceinline__ Piece of_lane(int lane) const {
    Piece o;
#pragma unroll
    for (int q = 0; q < N; ++q) o.w[q / 4][q % 4] = __shfl(w[q / 4][q % 4], lane, 64);
    return o;
  }
};
// N table values, or one for every two
template <int N> __device__ __forceinline__ void load_table(float (&v)[N], const float* p) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int g = 0; g < N / 4; ++g) {
      const f32x4 x = reinterpret_cast<const f32x4*>(p)[g];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[4 * g + q] = x[q];
    }
  } else {
    const f32x2 x = *reinterpret_cast<const f32x2*>(p);
    v[0] = x[0];
    v[1] = x[1];
  }
}

// ---- the turn, with or without a cache behind it ----------------------------------------------------------
// A wave has one token at a time and walks its head rows, 64 / lanes of them next to each other in memory per access and kAtOnce
// accesses in flight.  (A wave over as many tokens instead, a head
// row of each, moves 256-byte pieces: 40960 tokens of 32 + 4 heads 142 us, as it is 124.)
template <class E, int N, int CACHE /* 0: none, 1: elements as they are, 2: 8-bit blocks */>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a, int lanes, int heads_per_block) {
  const int lane = static_cast<int>(threadIdx.x) & 63, chunk = lane & (lanes - 1), sub = lane / lanes, abreast = 64 / lanes;
  if (chunk * N >= a.D) return;                        // lanes of the power of two that a head row has no elements for
  const int half = a.rot / 2;
  const bool turned = chunk * N < a.rot, first = chunk * N < half;
  const int partner = !turned ? lane : first ? lane + half / N : lane - half / N;
  const int turned_rows = a.Hq + a.Hk, rows = turned_rows + a.Hv;
  const int h0 = blockIdx.y * heads_per_block, h1 = min(rows, h0 + heads_per_block);

  for (long t = static_cast<long>(blockIdx.x) * kWaves + wave_of_block(); t < a.T; t += static_cast<long>(gridDim.x) * kWaves) {
    float co[N], si[N];
    if (turned && h0 < turned_rows) {
      const int p = min(max(a.positions[t], 0), a.n_pos - 1);
      if (a.interleaved) {
        const long at = static_cast<long>(p) * half + chunk * (N / 2);
        float c[N / 2], s[N / 2];
        load_table(c, a.cos + at);
        load_table(s, a.sin + at);
#pragma unroll
        for (int q = 0; q < N; ++q) {
          co[q] = c[q / 2];
          si[q] = (q % 2 == 0) == (a.back != 0) ? s[q / 2] : -s[q / 2];
        }
      } else {
        const long at = static_cast<long>(p) * half + (first ? chunk * N : chunk * N - half);
        load_table(co, a.cos + at);
        load_table(si, a.sin + at);
#pragma unroll
        for (int q = 0; q < N; ++q) si[q] = first == (a.back != 0) ? si[q] : -si[q];
      }
    } else {
#pragma unroll
      for (int q = 0; q < N; ++q) { co[q] = 1.0f; si[q] = 0.0f; }
    }
    long slot = -1;
    if (CACHE != 0 && h1 > a.Hq) {
      slot = a.slots[t];
      if (slot >= static_cast<long>(a.cache.pages) * a.cache.page_size) slot = -1;
    }
    const int page_shift = CACHE != 0 ? __builtin_ctz(a.cache.page_size) : 0;
    const long page = slot >> page_shift, place = slot & (a.cache.page_size - 1);

    for (int h = h0 + sub; h < h1; h += abreast * kAtOnce) {
      Piece<E, N> x[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int i = h + u * abreast;
        if (i >= h1) break;
        const bool is_q = i < a.Hq, is_v = i >= turned_rows;
        const E* src = static_cast<const E*>(is_q ? a.q : is_v ? a.v : a.k);
        const long st = is_q ? a.q_stride_t : is_v ? a.v_stride_t : a.k_stride_t, sh = is_q ? a.q_stride_h : is_v ? a.v_stride_h : a.k_stride_h;
        x[u].load(src + t * st + (is_q ? i : is_v ? i - turned_rows : i - a.Hq) * sh + chunk * N);
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int i = h + u * abreast;
        if (i >= h1) break;
        const bool is_q = i < a.Hq, is_v = i >= turned_rows;
        float y[N];
        x[u].get(y);
        if (!is_v) {
          float other[N];
          if (a.interleaved) {
#pragma unroll
            for (int q = 0; q < N; ++q) other[q] = y[q ^ 1];
          } else {
            x[u].of_lane(partner).get(other);
          }
          if (turned) {
#pragma clang fp contract(off)
#pragma unroll
            for (int q = 0; q < N; ++q) {
              const float own = y[q] * co[q], turn = other[q] * si[q];
              y[q] = own + turn;
            }
          }
        }
        Piece<E, N> o = x[u];
        if (!is_v && turned) o.set(y);
        if (CACHE == 0 || is_q) {
          E* dst = static_cast<E*>(is_q ? a.q_out : a.k_out);
          const long st = is_q ? a.qo_stride_t : a.ko_stride_t, sh = is_q ? a.qo_stride_h : a.ko_stride_h;
          o.store(dst + t * st + (is_q ? i : i - a.Hq) * sh + chunk * N);
        } else {
          const long row = static_cast<long>(is_v ? i - turned_rows : i - a.Hq) * a.cache.page_size + place;
          void* base = is_v ? a.cache.v : a.cache.k;
          if (CACHE == 1) {
            if (slot >= 0) o.store(static_cast<E*>(base) + page * a.cache.page_stride + row * a.D + chunk * N);
          } else if constexpr (CACHE == 2) {
            float amax = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) amax = fmaxf(amax, fabsf(y[q]));
            amax = quad_max(amax);                     // four lanes hold the 32 elements of a block
            const uint32_t code = mx_scale_code(amax);
            const uint2 w = mx_encode8(y, mx_inverse_scale(code));
            if (slot >= 0) {
              __builtin_nontemporal_store(u32x2{w.x, w.y}, reinterpret_cast<u32x2*>(static_cast<uint8_t*>(base) + page * a.cache.page_stride + row * a.D + chunk * 8));
              if ((chunk & 3) == 0)
                static_cast<uint8_t*>(is_v ? a.cache.v_scales : a.cache.k_scales)[page * a.cache.scale_page_stride + row * (a.D / 32) + chunk / 4] =
                    static_cast<uint8_t>(code);
            }
          }
        }
      }
    }
  }
}

int lanes_of_row(int D, int n) {
  int lanes = 1;
  while (lanes * n < D) lanes *= 2;
  return lanes;
}

template <class E, int N, int CACHE> void launch_rotate(const char* name, const RotateArgs& a) {
  const int lanes = lanes_of_row(a.D, N), step = 64 / lanes * kAtOnce, rows = a.Hq + a.Hk + a.Hv;
  const int bx = static_cast<int>(a.T / kWaves + (a.T % kWaves != 0)), gx = bx < kMaxBlocksX ? bx : kMaxBlocksX;
  // heads are cut into as many blocks as it takes to have kBlocksWanted workgroups; a block is a multiple of what a wave has in flight
  const int want = ceil_div(kBlocksWanted, gx), most = ceil_div(rows, step), cut = want < most ? want : most;
  const int heads = ceil_div(ceil_div(rows, cut), step) * step;
  MOE_LAUNCH(name, (rotate_kernel<E, N, CACHE>), dim3(gx, ceil_div(rows, heads)), dim3(kThreads), 0, a.stream, a, lanes, heads);
}

// ---- back from the pages ----------------------------------------------------------------------------------
// Output row r belongs to the sequence b with row_start[b] <= r < row_start[b + 1] and is its token first[b] + r - row_start[b].
// A wave has 64 / lanes consecutive rows, a row per group of `lanes` lanes, and walks the heads, kAtOnce in flight: consecutive tokens of one head
// lie next to each other in a page, so its reads are contiguous, and its stores whole head rows.
// (A wave over one to eight rows with the heads abreast: 52949 rows of 4 heads 40 to 50 us, as it is 38.)
template <int KIND /* MOE_F32, MOE_BF16 or MOE_MX8 */>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheReadArgs a, int lanes, int heads_per_block) {
  typedef std::conditional_t<KIND == MOE_F32, float, bf16_t> E;
  constexpr int N = 16 / sizeof(E);
  const int lane = static_cast<int>(threadIdx.x) & 63, chunk = lane & (lanes - 1), sub = lane / lanes, abreast = 64 / lanes, D = a.cache.dim, H = a.cache.heads;
  const int h0 = blockIdx.y * heads_per_block, h1 = min(2 * H, h0 + heads_per_block);   // keys, then values
  const int page_shift = __builtin_ctz(a.cache.page_size);
  const long held = static_cast<long>(a.max_pages) << page_shift;
  for (long r0 = (static_cast<long>(blockIdx.x) * kWaves + wave_of_block()) * abreast; r0 < a.rows; r0 += static_cast<long>(gridDim.x) * kWaves * abreast) {
    // the last b with row_start[b] <= r0, 64 candidates at a time; a later row of the wave is then a step or two further
    int b = 0;
    for (int count = a.B; count > 1;) {
      const int step = (count + 63) / 64;
      const bool before = lane * step < count && a.row_start[b + lane * step] <= r0;
      const int k = max(__builtin_popcountll(__ballot(before)) - 1, 0);
      b += k * step;
      count = min(step, count - k * step);
    }
    const long r = r0 + sub;
    if (chunk * N >= D || r >= a.rows) continue;
    long begin = a.row_start[b], end = a.row_start[b + 1];
    while (r >= end && b + 1 < a.B) {
      begin = end;
      end = a.row_start[++b + 1];
    }
    if (r < begin || r >= end) continue;               // rows that no sequence has stay as they are
    const long t = r - begin + (a.first ? a.first[b] : 0);
    int page = t >= 0 && t < held ? a.block_table[static_cast<long>(b) * a.max_pages + (t >> page_shift)] : -1;
    if (page >= a.cache.pages) page = -1;
    const int at = static_cast<int>(t & (a.cache.page_size - 1));
    const long place = page * a.cache.page_stride + static_cast<long>(at) * D + chunk * N;
    const long scale_place = page * a.cache.scale_page_stride + static_cast<long>(at) * (D / 32) + chunk / 4;
    for (int h = h0; h < h1; h += kAtOnce) {
      Piece<E, N> x[kAtOnce];
      u32x2 code[kAtOnce];
      uint32_t scale[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (h + u >= h1) break;
        const bool is_v = h + u >= H;
        const long head = static_cast<long>(is_v ? h + u - H : h + u) * a.cache.page_size;
        const void* base = is_v ? a.cache.v : a.cache.k;
        if (KIND == MOE_MX8) {
          code[u] = u32x2{0u, 0u};
          scale[u] = 0u;
          if (page >= 0) {
            code[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(base) + place + head * D));
            scale[u] = static_cast<const uint8_t*>(is_v ? a.cache.v_scales : a.cache.k_scales)[scale_place + head * (D / 32)];
          }
        } else {
          const float z[N] = {};
          x[u].set(z);
          if (page >= 0) x[u].load(static_cast<const E*>(base) + place + head * D);
        }
      }
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        if (h + u >= h1) break;
        const bool is_v = h + u >= H;
        if constexpr (KIND == MOE_MX8) {
          // exact in bf16 down to its smallest numbers
          const float sc = mx_scale(scale[u]);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            x[u].w[2 * q] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[u][q], sc, false));
            x[u].w[2 * q + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[u][q], sc, true));
          }
        }
        E* dst = static_cast<E*>(is_v ? a.v_out : a.k_out);
        x[u].store(dst + (r * H + (is_v ? h + u - H : h + u)) * D + chunk * N);
      }
    }
  }
}

template <int KIND> void launch_read(const CacheReadArgs& a) {
  const int lanes = lanes_of_row(a.cache.dim, KIND == MOE_F32 ? 4 : 8), per_block = kWaves * (64 / lanes), heads = 2 * a.cache.heads;
  const int bx = a.rows / per_block + (a.rows % per_block != 0), gx = bx < kMaxBlocksX ? bx : kMaxBlocksX;
  const int want = ceil_div(kBlocksWanted, gx), most = ceil_div(heads, kAtOnce), cut = want < most ? want : most;
  const int hpb = ceil_div(ceil_div(heads, cut), kAtOnce) * kAtOnce;
  MOE_LAUNCH("kv_cache_read", (cache_read_kernel<KIND>), dim3(gx, ceil_div(heads, hpb)), dim3(kThreads), 0, a.stream, a, lanes, hpb);
}

// ---- the table of cosines and sines -----------------------------------------------------------------------
// The angle of position p is formed and reduced in 64 bits: in 32 bits its error would be p 2^-24, a visible part of a turn from
// some ten thousand positions on.  Bound by that arithmetic: 163840 positions of 64 pairs 43 us (84 MB), 40960 14 us.
__global__ __launch_bounds__(kThreads) void rope_table_kernel(const double* __restrict__ freq, long total, int half, double amplitude,
                                                              float* __restrict__ cos_out, float* __restrict__ sin_out) {
  for (long i = static_cast<long>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<long>(gridDim.x) * kThreads) {
    double s, c;
    ::sincos(static_cast<double>(i / half) * freq[i % half], &s, &c);
    cos_out[i] = static_cast<float>(c * amplitude);
    sin_out[i] = static_cast<float>(s * amplitude);
  }
}

bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }
bool strides_ok(int dtype, int64_t t, int64_t h) { const int n = 16 / elem_size(dtype); return t % n == 0 && h % n == 0; }

int32_t check_heads(const char* who, int dtype, int T, int D, int rot) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
  MOE_REQUIRE(T >= 0 && D > 0 && rot >= 0 && rot <= D, MOE_ERR_INVALID_ARG, "%s: need T >= 0, D > 0 and 0 <= rot <= D (T=%d D=%d rot=%d)", who, T, D, rot);
  MOE_REQUIRE(D % 8 == 0 && D <= 512 && rot % 16 == 0, MOE_ERR_UNSUPPORTED, "%s: D=%d must be a multiple of 8 up to 512 and rot=%d one of 16", who, D, rot);
  return MOE_OK;
}

int32_t rope(const char* who, const char* name, int back, const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k, int64_t k_stride_t,
             int64_t k_stride_h, int dtype, int T, int Hq, int Hk, int D, int rot, const int32_t* positions, const float* cos, const float* sin,
             int n_pos, int interleaved, void* q_out, int64_t qo_stride_t, int64_t qo_stride_h, void* k_out, int64_t ko_stride_t, int64_t ko_stride_h,
             void* stream) {
  if (int32_t rc = check_heads(who, dtype, T, D, rot)) return rc;
  MOE_REQUIRE(Hq >= 0 && Hk >= 0 && Hq + static_cast<int64_t>(Hk) > 0 && Hq + static_cast<int64_t>(Hk) <= 65536, MOE_ERR_INVALID_ARG, "%s: heads Hq=%d Hk=%d", who, Hq, Hk);
  if (T == 0) return MOE_OK;
  MOE_REQUIRE((Hq == 0 || (q && q_out)) && (Hk == 0 || (k && k_out)), MOE_ERR_INVALID_ARG, "%s: null pointer", who);
  MOE_REQUIRE(rot == 0 || (positions && cos && sin && n_pos > 0), MOE_ERR_INVALID_ARG, "%s: a rotation needs positions and a table (n_pos=%d)", who, n_pos);
  MOE_REQUIRE(aligned16(q) && aligned16(k) && aligned16(q_out) && aligned16(k_out) && aligned16(cos) && aligned16(sin), MOE_ERR_INVALID_ARG,
              "%s: tensors must be 16-byte aligned", who);
  MOE_REQUIRE((Hq == 0 || (strides_ok(dtype, q_stride_t, q_stride_h) && strides_ok(dtype, qo_stride_t, qo_stride_h))) &&
              (Hk == 0 || (strides_ok(dtype, k_stride_t, k_stride_h) && strides_ok(dtype, ko_stride_t, ko_stride_h))), MOE_ERR_INVALID_ARG,
              "%s: strides must be multiples of 16 bytes", who);
  RotateArgs a{};
  a.q = q; a.q_stride_t = q_stride_t; a.q_stride_h = q_stride_h; a.k = k; a.k_stride_t = k_stride_t; a.k_stride_h = k_stride_h;
  a.T = T; a.Hq = Hq; a.Hk = Hk; a.Hv = 0; a.D = D; a.rot = rot; a.positions = positions; a.cos = cos; a.sin = sin; a.n_pos = n_pos;
  a.interleaved = interleaved != 0; a.back = back; a.q_out = q_out; a.qo_stride_t = qo_stride_t; a.qo_stride_h = qo_stride_h;
  a.k_out = k_out; a.ko_stride_t = ko_stride_t; a.ko_stride_h = ko_stride_h; a.stream = static_cast<hipStream_t>(stream);
  begin_call(who, a.stream);
  if (dtype == MOE_BF16) launch_rotate<bf16_t, 8, 0>(name, a);
  else if (D <= 256) launch_rotate<float, 4, 0>(name, a);
  else launch_rotate<float, 8, 0>(name, a);
  return end_call();
}

}  // namespace

int32_t check_cache(const char* who, const moe_kv_cache_t* c) {
  MOE_REQUIRE(c, MOE_ERR_INVALID_ARG, "%s: null cache", who);
  MOE_REQUIRE(c->dtype == MOE_F32 || c->dtype == MOE_BF16 || c->dtype == MOE_MX8, MOE_ERR_UNSUPPORTED, "%s: unknown dtype %d of the cache", who, c->dtype);
  MOE_REQUIRE(c->pages > 0 && c->heads > 0 && c->page_size > 0 && c->dim > 0, MOE_ERR_INVALID_ARG, "%s: cache of %d pages, %d heads, %d tokens a page, dim %d",
              who, c->pages, c->heads, c->page_size, c->dim);
  MOE_REQUIRE(c->heads <= 1024, MOE_ERR_UNSUPPORTED, "%s: %d heads in the cache, at most 1024", who, c->heads);
  MOE_REQUIRE(power_of_two(c->page_size) && c->page_size >= 16 && c->page_size <= 4096, MOE_ERR_UNSUPPORTED,
              "%s: page_size=%d must be a power of two from 16 to 4096", who, c->page_size);
  MOE_REQUIRE(c->dim == 64 || c->dim == 128 || c->dim == 192 || c->dim == 256, MOE_ERR_UNSUPPORTED, "%s: head dim %d is not 64, 128, 192 or 256", who, c->dim);
  const int64_t rows = static_cast<int64_t>(c->heads) * c->page_size;
  const int per16 = c->dtype == MOE_F32 ? 4 : c->dtype == MOE_BF16 ? 8 : 16;
  MOE_REQUIRE(c->page_stride >= rows * c->dim && c->page_stride % per16 == 0, MOE_ERR_INVALID_ARG, "%s: page_stride=%lld is below a page's %lld elements or no multiple of 16 bytes",
              who, static_cast<long long>(c->page_stride), static_cast<long long>(rows * c->dim));
  MOE_REQUIRE(c->k && c->v && aligned16(c->k) && aligned16(c->v), MOE_ERR_INVALID_ARG, "%s: cache pointers must be given and 16-byte aligned", who);
  if (c->dtype == MOE_MX8) {
    MOE_REQUIRE(c->k_scales && c->v_scales && aligned16(c->k_scales) && aligned16(c->v_scales), MOE_ERR_INVALID_ARG,
                "%s: an 8-bit cache needs its scales, 16-byte aligned", who);
    MOE_REQUIRE(c->scale_page_stride >= rows * (c->dim / 32) && c->scale_page_stride % 16 == 0, MOE_ERR_INVALID_ARG,
                "%s: scale_page_stride=%lld is below a page's %lld scales or no multiple of 16", who, static_cast<long long>(c->scale_page_stride),
                static_cast<long long>(rows * (c->dim / 32)));
  }
  return MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" int32_t moe_rope_table(const double* freq, int n_pos, int half, double amplitude, float* cos, float* sin, void* stream) {
  MOE_REQUIRE(n_pos >= 0 && half > 0, MOE_ERR_INVALID_ARG, "rope_table: need n_pos >= 0 and half > 0 (n_pos=%d half=%d)", n_pos, half);
  if (n_pos == 0) return MOE_OK;
  MOE_REQUIRE(freq && cos && sin && aligned16(freq) && aligned16(cos) && aligned16(sin), MOE_ERR_INVALID_ARG, "rope_table: null or misaligned pointer");
  const long total = static_cast<long>(n_pos) * half, blocks = (total + kThreads - 1) / kThreads;
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_rope_table", st);
  MOE_LAUNCH("rope_table", rope_table_kernel, dim3(static_cast<unsigned>(blocks < kMaxBlocksX ? blocks : kMaxBlocksX)), dim3(kThreads), 0, st, freq, total, half,
             amplitude, cos, sin);
  return end_call();
}

extern "C" int32_t moe_rope_fwd(const void* q, int64_t q_stride_t, int64_t q_stride_h, const void* k, int64_t k_stride_t, int64_t k_stride_h, int dtype,
                                int T, int Hq, int Hk, int D, int rot, const int32_t* positions, const float* cos, const float* sin, int n_pos,
                                int interleaved, void* q_out, int64_t qo_stride_t, int64_t qo_stride_h, void* k_out, int64_t ko_stride_t,
                                int64_t ko_stride_h, void* stream) {
  return rope("moe_rope_fwd", "rope_fwd", 0, q, q_stride_t, q_stride_h, k, k_stride_t, k_stride_h, dtype, T, Hq, Hk, D, rot, positions, cos, sin, n_pos,
              interleaved, q_out, qo_stride_t, qo_stride_h, k_out, ko_stride_t, ko_stride_h, stream);
}

extern "C" int32_t moe_rope_bwd(const void* dq, int64_t q_stride_t, int64_t q_stride_h, const void* dk, int64_t k_stride_t, int64_t k_stride_h, int dtype,
                                int T, int Hq, int Hk, int D, int rot, const int32_t* positions, const float* cos, const float* sin, int n_pos,
                                int interleaved, void* dq_in, int64_t qo_stride_t, int64_t qo_stride_h, void* dk_in, int64_t ko_stride_t,
                                int64_t ko_stride_h, void* stream) {
  return rope("moe_rope_bwd", "rope_bwd", 1, dq, q_stride_t, q_stride_h, dk, k_stride_t, k_stride_h, dtype, T, Hq, Hk, D, rot, positions, cos, sin, n_pos,
              interleaved, dq_in, qo_stride_t, qo_stride_h, dk_in, ko_stride_t, ko_stride_h, stream);
}

extern "C" int32_t moe_kv_cache_write(const moe_kv_cache_t* cache, const void* k, int64_t k_stride_t, int64_t k_stride_h, const void* v,
                                      int64_t v_stride_t, int64_t v_stride_h, int T, const int64_t* slots, const void* q, int64_t q_stride_t,
                                      int64_t q_stride_h, int Hq, int rot, const int32_t* positions, const float* cos, const float* sin, int n_pos,
                                      int interleaved, void* q_out, int64_t qo_stride_t, int64_t qo_stride_h, void* stream) {
  if (int32_t rc = check_cache("kv_cache_write", cache)) return rc;
  const int dtype = cache->dtype == MOE_F32 ? MOE_F32 : MOE_BF16;
  if (int32_t rc = check_heads("kv_cache_write", dtype, T, cache->dim, rot)) return rc;
  MOE_REQUIRE(Hq >= 0 && Hq <= 65536, MOE_ERR_INVALID_ARG, "kv_cache_write: Hq=%d", Hq);
  if (T == 0) return MOE_OK;
  MOE_REQUIRE(k && v && slots && (Hq == 0 || (q && q_out)), MOE_ERR_INVALID_ARG, "kv_cache_write: null pointer");
  MOE_REQUIRE(rot == 0 || (positions && cos && sin && n_pos > 0), MOE_ERR_INVALID_ARG, "kv_cache_write: a rotation needs positions and a table (n_pos=%d)", n_pos);
  MOE_REQUIRE(aligned16(k) && aligned16(v) && aligned16(q) && aligned16(q_out) && aligned16(cos) && aligned16(sin), MOE_ERR_INVALID_ARG,
              "kv_cache_write: tensors must be 16-byte aligned");
  MOE_REQUIRE(strides_ok(dtype, k_stride_t, k_stride_h) && strides_ok(dtype, v_stride_t, v_stride_h) &&
              (Hq == 0 || (strides_ok(dtype, q_stride_t, q_stride_h) && strides_ok(dtype, qo_stride_t, qo_stride_h))), MOE_ERR_INVALID_ARG,
              "kv_cache_write: strides must be multiples of 16 bytes");
  RotateArgs a{};
  a.q = q; a.q_stride_t = q_stride_t; a.q_stride_h = q_stride_h; a.k = k; a.k_stride_t = k_stride_t; a.k_stride_h = k_stride_h;
  a.v = v; a.v_stride_t = v_stride_t; a.v_stride_h = v_stride_h;
  a.T = T; a.Hq = Hq; a.Hk = a.Hv = cache->heads; a.D = cache->dim; a.rot = rot; a.positions = positions; a.cos = cos; a.sin = sin; a.n_pos = n_pos;
  a.interleaved = interleaved != 0; a.q_out = q_out; a.qo_stride_t = qo_stride_t; a.qo_stride_h = qo_stride_h;
  a.slots = slots; a.cache = *cache; a.stream = static_cast<hipStream_t>(stream);
  begin_call("moe_kv_cache_write", a.stream);
  if (cache->dtype == MOE_F32) launch_rotate<float, 4, 1>("kv_cache_write", a);
  else if (cache->dtype == MOE_BF16) launch_rotate<bf16_t, 8, 1>("kv_cache_write", a);
  else launch_rotate<bf16_t, 8, 2>("kv_cache_write", a);
  return end_call();
}

extern "C" int32_t moe_kv_cache_read(const moe_kv_cache_t* cache, const int32_t* block_table, int max_pages, const int32_t* row_start,
                                     const int32_t* first, int B, int rows, void* k_out, void* v_out, void* stream) {
  if (int32_t rc = check_cache("kv_cache_read", cache)) return rc;
  MOE_REQUIRE(B >= 0 && rows >= 0 && max_pages >= 0, MOE_ERR_INVALID_ARG, "kv_cache_read: need B, rows, max_pages >= 0 (B=%d rows=%d max_pages=%d)", B, rows, max_pages);
  if (B == 0 || rows == 0) return MOE_OK;
  MOE_REQUIRE(row_start && k_out && v_out && (max_pages == 0 || block_table), MOE_ERR_INVALID_ARG, "kv_cache_read: null pointer");
  MOE_REQUIRE(aligned16(k_out) && aligned16(v_out), MOE_ERR_INVALID_ARG, "kv_cache_read: tensors must be 16-byte aligned");
  CacheReadArgs a{*cache, block_table, row_start, first, k_out, v_out, max_pages, B, rows, static_cast<hipStream_t>(stream)};
  begin_call("moe_kv_cache_read", a.stream);
  if (cache->dtype == MOE_F32) launch_read<MOE_F32>(a);
  else if (cache->dtype == MOE_BF16) launch_read<MOE_BF16>(a);
  else launch_read<MOE_MX8>(a);
  return end_call();
}
