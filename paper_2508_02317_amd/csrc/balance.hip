// The router's balance loss and z loss, with the counts per expert, and their gradient.  Over the n tokens that are valid, with p = softmax(z[t, :]),
// c_e the number of their (token, slot) pairs that chose expert e and P_e = 1/n sum_t p[t, e]:
//
//     L_b = sum_e s_e P_e,  s_e = E c_e / (k n) (1 where all experts are chosen alike);      L_z = 1/n sum_t lse_t^2,  lse_t = log sum_e exp z[t, e]
//     dz[t, e] = p[t, e] ( a/n (s_e - sum_e' s_e' p[t, e']) + b 2/n lse_t )   for a L_b + b L_z; the counts are constants
//
// Bound by HBM and by launches: the logits are read once by each pass, the gradient (and what it is added to) once more.  A row belongs to `lanes` lanes of a
// wave, so that several short rows lie side by side, and a lane has the same columns of all its rows: the sums over tokens stay in its registers.  They go over the
// waves through LDS, as rows of the workspace to a second launch, and every step adds in a fixed order; counts are whole numbers, so their order is free.
// Measured, passes among others and in brackets the launches as the profiler sees each (together they come to more than a pass): 40960 tokens of 128 experts 23.1 to 23.3 us (9.0: 23 MB
// read, four fifths of the time are five dependent turns of a workgroup with the loads of one turn in flight; 5.8: one workgroup adds 256 rows, 260 KB; 9.8: 63 MB, 6.5 TB/s, part of it
// from the memory-side cache); 8192 tokens 14.7 to 16 (4.8, 6.0, 4.8); 8192 of 1024 experts 33.7; 256 tokens of 8 experts, which one workgroup does alone, are bound by the host's two
// calls, 8 to 9.5 (4.8 and 2.5).
#include "moe_common.h"
#include "pieces.h"

namespace moe {

namespace {

constexpr int kPieces = 2;                             // of 16 bytes that a lane has of a row, while 64 lanes suffice for it: 40960 tokens of 128 experts +1.3 us with four, +3.4 with one
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_at_4 __attribute__((ext_vector_type(4), aligned(4)));

// 512 workgroups forward: 40960 tokens +1.2 us, 8192 of 1024 experts +3 (twice the rows to add); 128: 8192 tokens -0.5, 40960 +3.6, 8192 of 512 experts +1.7
constexpr int kFwdThreads = 512, kFwdWaves = kFwdThreads / 64, kFwdBlocks = 256;
constexpr int kBwdThreads = 512, kBwdBlocks = 512;     // 1024 workgroups: 40960 tokens +1.5 us, 8192 of 1024 experts +4
constexpr size_t kHeadBytes = 512;                     // of the workspace: the join's counter and losses
constexpr int kJoinThreads = 1024, kJoinLanes = 32;    // lanes of a row of sums, at most: 16 and 8 (more workgroups, and their counter) +0.4 and +1.1 us at 128 experts

struct FwdArgs {
  const float* logits;
  const int32_t* topk_idx;
  const uint8_t* valid;                                // or null
  float *losses, *importance, *lse;
  int32_t* counts;
  int T, E, k, lanes, row;                             // row: E rounded up to whole pieces
  Divisor per_token;                                   // k
  // workspace: sums and counts [blocks][row], z and n [blocks], the join's losses and its counter
  float *sum_of, *z_of;
  int32_t *count_of, *n_of;
  double* loss_of;
  uint32_t* joined;
};
struct BwdArgs {
  const float* logits;
  const int32_t* counts;
  const float* lse;
  const uint8_t* valid;
  const float *dlosses, *add;                          // or null
  float* dlogits;
  int T, E, k, lanes;
  float balance, z;
};

// Four consecutive elements of a row from column e on, where the row has them.  Rows of E elements start at multiples of 4 bytes, which is all that a
// 16-byte access needs.  (The logits have just been written by the router's product, the gradient goes to its backward product: loads pass through the caches.)
// Loads are in straight-line code, at places that exist, and nothing touches what they bring before it is used: a load behind a branch, or one whose result
// is masked at once, is waited for there, and nothing would be in flight from one turn to the next.
// TAIL: E is no multiple of four.  A piece that would pass the row's end is read from the last four elements and moved into place when it is used.
template <bool TAIL> __device__ __forceinline__ f32x4 fetch(const float* row, int e, int E) {
  if (TAIL && E < 4) return f32x4{row[0], row[min(1, E - 1)], row[min(2, E - 1)], 0.0f};
  return *reinterpret_cast<const f32x4_at_4*>(row + min(e, E - 4));
}
template <bool TAIL> __device__ __forceinline__ void place(float (&v)[4], const f32x4& x, int e, int E, float beyond) {
  const int shift = TAIL && E < 4 ? e : e - min(e, E - 4);
  if (TAIL) {
    v[0] = shift == 0 ? x[0] : shift == 1 ? x[1] : shift == 2 ? x[2] : shift == 3 ? x[3] : beyond;
    v[1] = shift == 0 ? x[1] : shift == 1 ? x[2] : shift == 2 ? x[3] : beyond;
    v[2] = shift == 0 ? x[2] : shift == 1 ? x[3] : beyond;
    v[3] = shift == 0 ? x[3] : beyond;
    if (E < 4) {
#pragma unroll
      for (int q = 1; q < 4; ++q)
        if (q >= E) v[q] = beyond;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = shift == 0 ? x[q] : beyond;
  }
}
template <bool TAIL> __device__ __forceinline__ void store(const float (&v)[4], float* row, int e, int E) {
  if (!TAIL || e + 4 <= E) {
    __builtin_nontemporal_store(f32x4_at_4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_at_4*>(row + e));
  } else {
#pragma unroll
    for (int q = 0; q < 3; ++q)
      if (e + q < E) row[e + q] = v[q];
  }
}

// exp of a difference of logits that is near or below 0, by the hardware's power of two: the product's rounding is an error of 2^-24 |x|, as the
// difference's own is, in probabilities that are the smaller the larger it is.  (With the library's expf, three times the instructions: 40960 tokens of 128 experts +1.6 us,
// 8192 of 1024 +2.2.  Outputs' errors against 64 bits 1.0e-7 with either.)
__device__ __forceinline__ float exp_near(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// Over the first WAVES waves of a workgroup; scratch: one of each of them, the result in thread 0
template <int WAVES> __device__ __forceinline__ double block_sum(double v, double* scratch) {
  if (static_cast<int>(threadIdx.x) < 64 * WAVES) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  }
  __syncthreads();
  double all = 0.0;
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < WAVES; ++i) all += scratch[i];
  }
  return all;
}

// What becomes of an expert's sums; returns its part of sum_e c_e P_e.
__device__ __forceinline__ double finish_expert(const FwdArgs& a, int e, float sum, int32_t count, int32_t n) {
  const float importance = sum / static_cast<float>(max(n, 1));
  a.importance[e] = importance;
  a.counts[e] = count;
  return static_cast<double>(count) * importance;
}
__device__ __forceinline__ void finish(const FwdArgs& a, double balance, double z, int32_t n) {
  const double many = max(n, 1);
  a.losses[0] = static_cast<float>(balance * a.E / (many * a.k));
  a.losses[1] = static_cast<float>(z / many);
  a.counts[a.E] = n;
}

// P pieces of four columns a lane.  ONE: the only workgroup, which needs no join.
template <int P, bool TAIL, bool ONE>
__global__ __launch_bounds__(kFwdThreads) void balance_fwd_kernel(FwdArgs a) {
  extern __shared__ char shared[];                     // [waves][row] sums, [row] counts
  __shared__ double scratch[kFwdWaves];
  __shared__ float z_wave[kFwdWaves];
  __shared__ int n_wave[kFwdWaves];
  float* sums = reinterpret_cast<float*>(shared);
  int32_t* counts = reinterpret_cast<int32_t*>(sums + kFwdWaves * a.row);
  const int l = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6, lane = l & (a.lanes - 1), group = static_cast<int>(threadIdx.x) / a.lanes;
  const int groups = kFwdThreads / a.lanes;
  const long step = static_cast<long>(gridDim.x) * groups;
  long t = static_cast<long>(blockIdx.x) * groups + group;
  // what is needed first is requested first: the rows of the first turn, this workgroup's share of the pairs, then the rows of each next turn
  f32x4 x[P];
  uint32_t on = 0;
  auto request = [&](long row) {
    const long r = min(row, a.T - 1l);
#pragma unroll
    for (int p = 0; p < P; ++p) x[p] = fetch<TAIL>(a.logits + r * a.E, (p * a.lanes + lane) * 4, a.E);
    on = a.valid ? a.valid[r] : 1u;
  };
  if (a.T > 0) request(t);
  for (int e = threadIdx.x; e < a.E; e += kFwdThreads) counts[e] = 0;
  {
    const long share = (a.T + static_cast<long>(gridDim.x) - 1) / gridDim.x, first = blockIdx.x * share * a.k, last = min(first + share * a.k, static_cast<long>(a.T) * a.k);
    long i = first + threadIdx.x;
    int e = i < last ? a.topk_idx[i] : -1;
    uint32_t counted = i < last && a.valid ? a.valid[divide(static_cast<uint32_t>(i), a.per_token)] : 1u;
    __syncthreads();
    while (i < last) {
      if (counted && e >= 0 && e < a.E) atomicAdd(&counts[e], 1);
      i += kFwdThreads;
      if (i >= last) break;
      e = a.topk_idx[i];
      if (a.valid) counted = a.valid[divide(static_cast<uint32_t>(i), a.per_token)];
    }
  }
  float acc[P][4], z_sum = 0.0f;
  int n = 0;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[p][q] = 0.0f;
  for (long base = static_cast<long>(blockIdx.x) * groups; base < a.T; base += step, t += step) {
    const bool there = t < a.T && on != 0;
    float e[P][4], top = -INFINITY;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      place<TAIL>(e[p], x[p], (p * a.lanes + lane) * 4, a.E, -INFINITY);
#pragma unroll
      for (int q = 0; q < 4; ++q) top = fmaxf(top, e[p][q]);
    }
    if (base + step < a.T) request(t + step);
    top = lanes_max(top, a.lanes);
    const float from = top == -INFINITY ? 0.0f : top;  // a row without a finite logit has no probabilities
    float total = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        e[p][q] = exp_near(e[p][q] - from);
        total += e[p][q];
      }
    total = lanes_sum(total, a.lanes);
    const float scale = total == 0.0f ? 0.0f : 1.0f / total, lse = there ? top + logf(total) : 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[p][q] += there ? e[p][q] * scale : 0.0f;   // padding may hold anything
    if (lane == 0 && t < a.T) {
      a.lse[t] = lse;
      n += there;
      z_sum += lse == -INFINITY ? 0.0f : lse * lse;
    }
  }
  // over the rows of a wave, then over the waves
  for (int o = a.lanes; o < 64; o *= 2) {
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[p][q] += __shfl_xor(acc[p][q], o, 64);
  }
  z_sum = wave_sum(z_sum);
  n = wave_sum_i(n);
  if (l < a.lanes) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int e = (p * a.lanes + lane) * 4;
      if (e < a.E) {
#pragma unroll
        for (int q = 0; q < 4; ++q) sums[wave * a.row + e + q] = acc[p][q];
      }
    }
  }
  if (l == 0) { z_wave[wave] = z_sum; n_wave[wave] = n; }
  __syncthreads();
  n = 0;
  z_sum = 0.0f;
  for (int w = 0; w < kFwdWaves; ++w) { n += n_wave[w]; z_sum += z_wave[w]; }
  double balance = 0.0;
  for (int e = threadIdx.x; e < a.E; e += kFwdThreads) {
    float sum = 0.0f;
    for (int w = 0; w < kFwdWaves; ++w) sum += sums[w * a.row + e];
    if (ONE) {
      balance += finish_expert(a, e, sum, counts[e], n);
    } else {
      a.sum_of[static_cast<long>(blockIdx.x) * a.row + e] = sum;
      a.count_of[static_cast<long>(blockIdx.x) * a.row + e] = counts[e];
    }
  }
  if (ONE) {
    balance = block_sum<kFwdWaves>(balance, scratch);
    if (threadIdx.x == 0) finish(a, balance, z_sum, n);
  } else if (threadIdx.x == 0) {
    a.z_of[blockIdx.x] = z_sum;
    a.n_of[blockIdx.x] = n;
    if (blockIdx.x == 0) *a.joined = 0;
  }
}

// The workgroups' rows added: `lanes` (a power of two up to kJoinLanes) lanes of four experts a workgroup, the rows dealt out to kJoinThreads / lanes runs, which are
// added over a wave and over the waves.  The last workgroup to end, by a counter that the launch before has cleared, adds the losses of all in the order of
// their numbers.
__global__ __launch_bounds__(kJoinThreads) void balance_join_kernel(FwdArgs a, int parts, int lanes) {
  constexpr int kWaves = kJoinThreads / 64;
  __shared__ float sums[kWaves][kJoinLanes * 4];
  __shared__ int32_t counts[kWaves][kJoinLanes * 4], n_all;
  constexpr int kSumWaves = kJoinLanes * 4 / 64;       // a thread for each of the workgroup's columns
  __shared__ double scratch[kSumWaves], z_all;
  const int l = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6, lane = l & (lanes - 1), runs = kJoinThreads / lanes;
  const int e = (blockIdx.x * lanes + lane) * 4;
  f32x4 sum = {};
  i32x4 count = {};
  int n = 0;
  double z = 0.0;
  if (wave == kWaves - 1) {                            // tokens and squares are the last wave's to sum, beside its columns
#pragma unroll
    for (int u = 0; u < kFwdBlocks / 64; ++u) {
      const int i = u * 64 + l;
      n += i < parts ? a.n_of[i] : 0;
      z += i < parts ? a.z_of[i] : 0.0f;
    }
  }
  if (e < a.E) {
#pragma unroll 8
    for (int i = static_cast<int>(threadIdx.x) / lanes; i < parts; i += runs) {
      const long at = static_cast<long>(i) * a.row + e;
      sum += *reinterpret_cast<const f32x4*>(a.sum_of + at);
      count += *reinterpret_cast<const i32x4*>(a.count_of + at);   // behind E, in a row's last piece, lies anything
    }
  }
  if (wave == kWaves - 1) {
    n = wave_sum_i(n);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o, 64);
    if (l == 0) { n_all = n; z_all = z; }
  }
  for (int o = lanes; o < 64; o *= 2)
#pragma unroll
    for (int q = 0; q < 4; ++q) { sum[q] += __shfl_xor(sum[q], o, 64); count[q] += __shfl_xor(count[q], o, 64); }
  if (l < lanes) {
#pragma unroll
    for (int q = 0; q < 4; ++q) { sums[wave][lane * 4 + q] = sum[q]; counts[wave][lane * 4 + q] = count[q]; }
  }
  __syncthreads();
  n = n_all;
  double balance = 0.0;
  const int mine = blockIdx.x * lanes * 4 + threadIdx.x;
  if (static_cast<int>(threadIdx.x) < lanes * 4 && mine < a.E) {
    float s = 0.0f;
    int32_t c = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { s += sums[w][threadIdx.x]; c += counts[w][threadIdx.x]; }
    balance = finish_expert(a, mine, s, c, n);
  }
  balance = block_sum<kSumWaves>(balance, scratch);
  if (threadIdx.x != 0) return;
  if (gridDim.x > 1) {
    __hip_atomic_store(&a.loss_of[blockIdx.x], balance, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__hip_atomic_fetch_add(a.joined, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 != gridDim.x) return;
    balance = 0.0;
    for (unsigned i = 0; i < gridDim.x; ++i) balance += __hip_atomic_load(&a.loss_of[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  finish(a, balance, z_all, n);
}

template <int P, bool TAIL, bool ADD>
__global__ __launch_bounds__(kBwdThreads) void balance_bwd_kernel(BwdArgs a) {
  const int lane = static_cast<int>(threadIdx.x) & (a.lanes - 1), group = static_cast<int>(threadIdx.x) / a.lanes, groups = kBwdThreads / a.lanes;
  const long step = static_cast<long>(gridDim.x) * groups;
  long t = static_cast<long>(blockIdx.x) * groups + group;
  f32x4 x[P], more[P];
  float lse_next;
  uint32_t on;
  auto request = [&](long row) {
    const long r = min(row, a.T - 1l);
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int e = (p * a.lanes + lane) * 4;
      x[p] = fetch<TAIL>(a.logits + r * a.E, e, a.E);
      if constexpr (ADD) more[p] = fetch<TAIL>(a.add + r * a.E, e, a.E);
    }
    lse_next = a.lse[r];
    on = a.valid ? a.valid[r] : 1u;
  };
  request(t);
  float share[P][4];
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int e = (p * a.lanes + lane) * 4 + q, count = a.counts[min(e, a.E)];
      share[p][q] = e < a.E ? static_cast<float>(count) : 0.0f;
    }
  const float many = static_cast<float>(max(a.counts[a.E], 1));
  const float to_balance = a.balance * (a.dlosses ? a.dlosses[0] : 1.0f) / many, to_z = 2.0f * a.z * (a.dlosses ? a.dlosses[1] : 1.0f) / many;
  const float per_pair = static_cast<float>(a.E) / static_cast<float>(a.k) / many;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int q = 0; q < 4; ++q) share[p][q] *= per_pair;
  for (long base = static_cast<long>(blockIdx.x) * groups; base < a.T; base += step, t += step) {
    const float lse = lse_next;
    const bool any = on != 0 && lse != -INFINITY;      // else the token does not count, or has no finite logit
    const float push = any ? to_balance : 0.0f, level = any ? lse * to_z : 0.0f;   // dlosses may be infinite or NaN
    float e[P][4], out[P][4], sums[2] = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * a.lanes + lane) * 4;
      place<TAIL>(e[p], x[p], c, a.E, -INFINITY);
      if constexpr (ADD) place<TAIL>(out[p], more[p], c, a.E, 0.0f);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        e[p][q] = any ? exp_near(e[p][q] - lse) : 0.0f;
        if constexpr (!ADD) out[p][q] = 0.0f;
        sums[0] += e[p][q];
        sums[1] += share[p][q] * e[p][q];
      }
    }
    if (base + step < a.T) request(t + step);
    // the sum of exp(z - lse) is 1 but for the rounding of lse, which dividing by it takes out of the probabilities
    const float total = lanes_sum(sums[0], a.lanes), scale = total == 0.0f ? 0.0f : 1.0f / total, mean = lanes_sum(sums[1], a.lanes) * scale;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * a.lanes + lane) * 4;
#pragma unroll
      for (int q = 0; q < 4; ++q) out[p][q] += e[p][q] * scale * ((share[p][q] - mean) * push + level);
      if (t < a.T && c < a.E) store<TAIL>(out[p], a.dlogits + t * a.E, c, a.E);
    }
  }
}

int fwd_blocks(int T, int E) {
  const int rows = kFwdThreads / split_columns(E, kPieces).lanes, n = T / rows + (T % rows != 0);
  return n < 1 ? 1 : n < kFwdBlocks ? n : kFwdBlocks;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int32_t check_balance(const char* who, int T, int E, int k) {
  MOE_REQUIRE(T >= 0 && E > 0 && k > 0, MOE_ERR_INVALID_ARG, "%s: need T >= 0, E > 0, k > 0 (T=%d E=%d k=%d)", who, T, E, k);
  MOE_REQUIRE(k <= E, MOE_ERR_INVALID_ARG, "%s: k=%d exceeds E=%d", who, k, E);
  MOE_REQUIRE(E <= kMaxExperts, MOE_ERR_UNSUPPORTED, "%s: E=%d above the built maximum %d", who, E, kMaxExperts);
  MOE_REQUIRE(k <= kMaxTopK, MOE_ERR_UNSUPPORTED, "%s: k=%d above the built maximum %d", who, k, kMaxTopK);
  MOE_REQUIRE(static_cast<int64_t>(T) * k <= INT32_MAX, MOE_ERR_UNSUPPORTED, "%s: T*k does not fit in int32", who);
  return MOE_OK;
}

template <class F> void with_pieces(int pieces, bool tail, F f) {
  auto tailed = [&](auto p) { if (tail) f(p, std::true_type{}); else f(p, std::false_type{}); };
  if (pieces == 1) tailed(std::integral_constant<int, 1>{});
  else if (pieces == 2) tailed(std::integral_constant<int, 2>{});
  else tailed(std::integral_constant<int, 4>{});       // 64 lanes of up to 1024 experts
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_balance_loss_fwd_workspace_bytes(int T, int E, int k) {
  (void)k;
  if (T < 0 || E <= 0 || E > kMaxExperts) return 0;
  const size_t blocks = fwd_blocks(T, E);
  return align_up(blocks * (2 * static_cast<size_t>(split_columns(E, kPieces).row) + 2) * 4, 16) + kHeadBytes;
}

extern "C" int32_t moe_balance_loss_fwd(const float* logits, const int32_t* topk_idx, const uint8_t* valid, int T, int E, int k, float* losses, int32_t* counts,
                                        float* importance, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_balance("balance_loss_fwd", T, E, k)) return rc;
  MOE_REQUIRE(losses && counts && importance && (T == 0 || (logits && topk_idx && lse)), MOE_ERR_INVALID_ARG, "balance_loss_fwd: null pointer");
  MOE_REQUIRE(aligned4(logits) && aligned4(topk_idx) && aligned4(losses) && aligned4(counts) && aligned4(importance) && aligned4(lse), MOE_ERR_INVALID_ARG,
              "balance_loss_fwd: tensors must be 4-byte aligned");
  const size_t need = moe_balance_loss_fwd_workspace_bytes(T, E, k);
  MOE_REQUIRE(ws && ws_bytes >= need && aligned16(ws), MOE_ERR_WORKSPACE, "balance_loss_fwd: workspace null, misaligned or smaller than %zu bytes", need);
  const ColumnSplit s = split_columns(E, kPieces);
  const int blocks = fwd_blocks(T, E);
  FwdArgs a{logits, topk_idx, valid, losses, importance, lse, counts, T, E, k, s.lanes, s.row, divisor(k), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
  a.joined = static_cast<uint32_t*>(ws);
  a.loss_of = reinterpret_cast<double*>(static_cast<char*>(ws) + 16);                 // of the join's workgroups
  static_assert(16 + kMaxExperts / kJoinLanes * sizeof(double) <= kHeadBytes);
  a.sum_of = reinterpret_cast<float*>(static_cast<char*>(ws) + kHeadBytes);
  a.count_of = reinterpret_cast<int32_t*>(a.sum_of + static_cast<size_t>(blocks) * s.row);
  a.z_of = reinterpret_cast<float*>(a.count_of + static_cast<size_t>(blocks) * s.row);
  a.n_of = reinterpret_cast<int32_t*>(a.z_of + blocks);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const size_t lds = (kFwdWaves + 1) * static_cast<size_t>(s.row) * 4;
  begin_call("moe_balance_loss_fwd", st);
  with_pieces(s.pieces, E % 4 != 0, [&](auto p, auto t) {
    constexpr int P = decltype(p)::value;
    constexpr bool TAIL = decltype(t)::value;
    if (blocks == 1) MOE_LAUNCH("balance_fwd", (balance_fwd_kernel<P, TAIL, true>), dim3(1), dim3(kFwdThreads), lds, st, a);
    else MOE_LAUNCH("balance_fwd", (balance_fwd_kernel<P, TAIL, false>), dim3(blocks), dim3(kFwdThreads), lds, st, a);
  });
  if (blocks > 1) {
    const int pieces = s.row / 4;
    int lanes = 1;
    while (lanes < pieces && lanes < kJoinLanes) lanes *= 2;
    MOE_LAUNCH("balance_join", balance_join_kernel, dim3(ceil_div(pieces, lanes)), dim3(kJoinThreads), 0, st, a, blocks, lanes);
  }
  return end_call();
}

extern "C" int32_t moe_balance_loss_bwd(const float* logits, const int32_t* counts, const float* lse, const uint8_t* valid, int T, int E, int k, float balance, float z,
                                        const float* dlosses, const float* add, float* dlogits, void* stream) {
  if (int32_t rc = check_balance("balance_loss_bwd", T, E, k)) return rc;
  if (T == 0) return MOE_OK;
  MOE_REQUIRE(logits && counts && lse && dlogits, MOE_ERR_INVALID_ARG, "balance_loss_bwd: null pointer");
  MOE_REQUIRE(aligned4(logits) && aligned4(counts) && aligned4(lse) && aligned4(dlosses) && aligned4(add) && aligned4(dlogits), MOE_ERR_INVALID_ARG,
              "balance_loss_bwd: tensors must be 4-byte aligned");
  const ColumnSplit s = split_columns(E, kPieces);
  BwdArgs a{logits, counts, lse, valid, dlosses, add, dlogits, T, E, k, s.lanes, balance, z};
  const int rows = kBwdThreads / s.lanes, blocks = T / rows + (T % rows != 0);
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_balance_loss_bwd", st);
  with_pieces(s.pieces, E % 4 != 0, [&](auto p, auto t) {
    constexpr int P = decltype(p)::value;
    constexpr bool TAIL = decltype(t)::value;
    const dim3 grid(blocks < kBwdBlocks ? blocks : kBwdBlocks);
    if (add) MOE_LAUNCH("balance_bwd", (balance_bwd_kernel<P, TAIL, true>), grid, dim3(kBwdThreads), 0, st, a);
    else MOE_LAUNCH("balance_bwd", (balance_bwd_kernel<P, TAIL, false>), grid, dim3(kBwdThreads), 0, st, a);
  });
  return end_call();
}
