// The router's balance loss and z loss, with the counts per expert, and their gradient.  Over the n tokens that are valid, with p = softmax(z[t, :]),
// c_e the number of their (token, slot) pairs that chose expert e and P_e = 1/n sum_t p[t, e]:
//
//     L_b = sum_e s_e P_e,  s_e = E c_e / (k n) (1 where all experts are chosen alike);      L_z = 1/n sum_t lse_t^2,  lse_t = log sum_e exp z[t, e]
//     dz[t, e] = p[t, e] ( a/n (s_e - sum_e' s_e' p[t, e']) + b 2/n lse_t )   for a L_b + b L_z; the counts are constants
//
// Bound by HBM: the logits are read once by each pass, the gradient (and what it is added to) once more.  A row belongs to `lanes` lanes of a wave, so
// that several short rows lie side by side, and a lane has the same columns of all its rows: the sums over tokens stay in its registers.  They go over the
// waves through LDS, as rows of the workspace to a second launch, and every step adds in a fixed order; counts are whole numbers, so their order is free.
#include "moe_common.h"
#include "pieces.h"

namespace moe {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kFwdThreads = 512, kFwdWaves = kFwdThreads / 64, kFwdBlocks = 256;
constexpr int kBwdThreads = 256, kBwdBlocks = 4096;
constexpr size_t kHeadBytes = 512;                     // of the workspace: the join's counter and losses
constexpr int kJoinThreads = 1024, kJoinLanes = 32;    // lanes of a row of sums, at most

struct FwdArgs {
  const float* logits;
  const int32_t* topk_idx;
  const uint8_t* valid;                                // or null
  float *losses, *importance, *lse;
  int32_t* counts;
  int T, E, k, lanes;
  Divisor per_token;                                   // k
  // workspace: sums and counts [blocks][E], z and n [blocks], the join's losses and its counter
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

template <int N> __device__ __forceinline__ void load(float (&v)[N], const float* p) {
  if constexpr (N == 4) {
    const f32x4 x = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = x[q];
  } else {
    v[0] = *p;
  }
}
template <int N> __device__ __forceinline__ void store(const float (&v)[N], float* p) {
  if constexpr (N == 4) __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4*>(p));
  else *p = v[0];
}

__device__ __forceinline__ double block_sum(double v, double* scratch) {   // scratch: one of each wave; the result in thread 0
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  double all = 0.0;
  if (threadIdx.x == 0)
    for (int i = 0; i < static_cast<int>(blockDim.x) >> 6; ++i) all += scratch[i];
  return all;
}

// What becomes of an expert's sums; returns its part of the balance loss.
__device__ __forceinline__ double finish_expert(const FwdArgs& a, int e, float sum, int32_t count, int32_t n) {
  const float many = static_cast<float>(max(n, 1)), importance = sum / many;
  a.importance[e] = importance;
  a.counts[e] = count;
  return static_cast<double>(count) * a.E / (static_cast<double>(a.k) * max(n, 1)) * importance;
}
__device__ __forceinline__ void finish(const FwdArgs& a, double balance, double z, int32_t n) {
  a.losses[0] = static_cast<float>(balance);
  a.losses[1] = static_cast<float>(z / max(n, 1));
  a.counts[a.E] = n;
}

// N columns a piece (4 where rows are whole pieces of 16 bytes), P pieces a lane.  ONE: the only workgroup, which needs no join.
template <int N, int P, bool ONE>
__global__ __launch_bounds__(kFwdThreads) void balance_fwd_kernel(FwdArgs a) {
  extern __shared__ char shared[];                     // [waves][E] sums, [E] counts
  __shared__ double scratch[kFwdWaves];
  __shared__ float z_wave[kFwdWaves];
  __shared__ int n_wave[kFwdWaves];
  float* sums = reinterpret_cast<float*>(shared);
  int32_t* counts = reinterpret_cast<int32_t*>(sums + kFwdWaves * a.E);
  const int l = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6, lane = l & (a.lanes - 1), group = static_cast<int>(threadIdx.x) / a.lanes;
  const int groups = kFwdThreads / a.lanes;
  const long step = static_cast<long>(gridDim.x) * groups;
  long t = static_cast<long>(blockIdx.x) * groups + group;
  // what is needed first is requested first: the rows of the first turn, this workgroup's share of the pairs, then the rows of each next turn
  float v[P][N];
  uint32_t on;
  auto fetch = [&](long row) {
    on = row < a.T ? a.valid ? a.valid[row] : 1u : 0u;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int e = (p * a.lanes + lane) * N;
#pragma unroll
      for (int q = 0; q < N; ++q) v[p][q] = -INFINITY;
      if (row < a.T && e < a.E) load(v[p], a.logits + row * a.E + e);
    }
  };
  fetch(t);
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
  float acc[P][N], z_sum = 0.0f;
  int n = 0;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int q = 0; q < N; ++q) acc[p][q] = 0.0f;
  for (long base = static_cast<long>(blockIdx.x) * groups; base < a.T; base += step, t += step) {
    const bool there = on != 0;
    float e[P][N], top = -INFINITY;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < N; ++q) {
        e[p][q] = there ? v[p][q] : -INFINITY;         // padding may hold anything
        top = fmaxf(top, e[p][q]);
      }
    if (base + step < a.T) fetch(t + step);
    top = lanes_max(top, a.lanes);
    const float from = top == -INFINITY ? 0.0f : top;  // a row without a finite logit has no probabilities
    float total = 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < N; ++q) {
        e[p][q] = expf(e[p][q] - from);
        total += e[p][q];
      }
    total = lanes_sum(total, a.lanes);
    const float scale = total == 0.0f ? 0.0f : 1.0f / total, lse = there ? top + logf(total) : 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < N; ++q) acc[p][q] += e[p][q] * scale;
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
      for (int q = 0; q < N; ++q) acc[p][q] += __shfl_xor(acc[p][q], o, 64);
  }
  z_sum = wave_sum(z_sum);
  n = wave_sum_i(n);
  if (l < a.lanes) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int e = (p * a.lanes + lane) * N;
      if (e < a.E) {
#pragma unroll
        for (int q = 0; q < N; ++q) sums[wave * a.E + e + q] = acc[p][q];
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
    for (int w = 0; w < kFwdWaves; ++w) sum += sums[w * a.E + e];
    if (ONE) {
      balance += finish_expert(a, e, sum, counts[e], n);
    } else {
      a.sum_of[static_cast<long>(blockIdx.x) * a.E + e] = sum;
      a.count_of[static_cast<long>(blockIdx.x) * a.E + e] = counts[e];
    }
  }
  if (ONE) {
    balance = block_sum(balance, scratch);
    if (threadIdx.x == 0) finish(a, balance, z_sum, n);
  } else if (threadIdx.x == 0) {
    a.z_of[blockIdx.x] = z_sum;
    a.n_of[blockIdx.x] = n;
    if (blockIdx.x == 0) *a.joined = 0;
  }
}

// The workgroups' rows added: `lanes` (a power of two up to kJoinLanes) lanes of N experts a workgroup, the rows dealt out to kJoinThreads / lanes runs, which are
// added over a wave and over the waves.  The last workgroup to end, by a counter that the launch before has cleared, adds the losses of all in the order of
// their numbers.
template <int N> __global__ __launch_bounds__(kJoinThreads) void balance_join_kernel(FwdArgs a, int parts, int lanes) {
  constexpr int kWaves = kJoinThreads / 64;
  __shared__ float sums[kWaves][kJoinLanes * N];
  __shared__ int32_t counts[kWaves][kJoinLanes * N], n_wave[kWaves];
  __shared__ double scratch[2][kWaves];
  const int l = static_cast<int>(threadIdx.x) & 63, wave = static_cast<int>(threadIdx.x) >> 6, lane = l & (lanes - 1), runs = kJoinThreads / lanes;
  const int e = (blockIdx.x * lanes + lane) * N;
  float sum[N] = {};
  int32_t count[N] = {};
  if (e < a.E) {
#pragma unroll 4
    for (int i = static_cast<int>(threadIdx.x) / lanes; i < parts; i += runs) {
      const long at = static_cast<long>(i) * a.E + e;
      if constexpr (N == 4) {
        const f32x4 s = *reinterpret_cast<const f32x4*>(a.sum_of + at);
        const i32x4 c = *reinterpret_cast<const i32x4*>(a.count_of + at);
#pragma unroll
        for (int q = 0; q < N; ++q) { sum[q] += s[q]; count[q] += c[q]; }
      } else {
        sum[0] += a.sum_of[at];
        count[0] += a.count_of[at];
      }
    }
  }
  int n = 0;
  double z = 0.0;
  for (int i = threadIdx.x; i < parts; i += kJoinThreads) { n += a.n_of[i]; z += a.z_of[i]; }
  for (int o = lanes; o < 64; o *= 2)
#pragma unroll
    for (int q = 0; q < N; ++q) { sum[q] += __shfl_xor(sum[q], o, 64); count[q] += __shfl_xor(count[q], o, 64); }
  if (l < lanes) {
#pragma unroll
    for (int q = 0; q < N; ++q) { sums[wave][lane * N + q] = sum[q]; counts[wave][lane * N + q] = count[q]; }
  }
  n = wave_sum_i(n);
  if (l == 0) n_wave[wave] = n;
  z = block_sum(z, scratch[0]);                        // its barrier stands before the reads below too
  n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) n += n_wave[w];
  double balance = 0.0;
  const int mine = blockIdx.x * lanes * N + threadIdx.x;
  if (static_cast<int>(threadIdx.x) < lanes * N && mine < a.E) {
    float s = 0.0f;
    int32_t c = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) { s += sums[w][threadIdx.x]; c += counts[w][threadIdx.x]; }
    balance = finish_expert(a, mine, s, c, n);
  }
  balance = block_sum(balance, scratch[1]);
  if (threadIdx.x != 0) return;
  if (gridDim.x > 1) {
    __hip_atomic_store(&a.loss_of[blockIdx.x], balance, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__hip_atomic_fetch_add(a.joined, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 != gridDim.x) return;
    balance = 0.0;
    for (unsigned i = 0; i < gridDim.x; ++i) balance += __hip_atomic_load(&a.loss_of[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  finish(a, balance, z, n);
}

template <int N, int P>
__global__ __launch_bounds__(kBwdThreads) void balance_bwd_kernel(BwdArgs a) {
  const int lane = static_cast<int>(threadIdx.x) & (a.lanes - 1), group = static_cast<int>(threadIdx.x) / a.lanes, groups = kBwdThreads / a.lanes;
  const long step = static_cast<long>(gridDim.x) * groups;
  long t = static_cast<long>(blockIdx.x) * groups + group;
  float v[P][N], more[P][N], lse;
  uint32_t on;
  auto fetch = [&](long row) {
    const bool inside = row < a.T;
    on = inside ? a.valid ? a.valid[row] : 1u : 0u;
    lse = inside ? a.lse[row] : 0.0f;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int e = (p * a.lanes + lane) * N;
#pragma unroll
      for (int q = 0; q < N; ++q) { v[p][q] = -INFINITY; more[p][q] = 0.0f; }
      if (inside && e < a.E) {
        load(v[p], a.logits + row * a.E + e);
        if (a.add) load(more[p], a.add + row * a.E + e);
      }
    }
  };
  fetch(t);
  const float many = static_cast<float>(max(a.counts[a.E], 1));
  const float to_balance = a.balance * (a.dlosses ? a.dlosses[0] : 1.0f) / many, to_z = 2.0f * a.z * (a.dlosses ? a.dlosses[1] : 1.0f) / many;
  const float per_pair = static_cast<float>(a.E) / static_cast<float>(a.k) / many;
  float share[P][N];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int e = (p * a.lanes + lane) * N;
#pragma unroll
    for (int q = 0; q < N; ++q) share[p][q] = 0.0f;
    if (e < a.E) {
      if constexpr (N == 4) {
        const i32x4 c = *reinterpret_cast<const i32x4*>(a.counts + e);
#pragma unroll
        for (int q = 0; q < N; ++q) share[p][q] = static_cast<float>(c[q]) * per_pair;
      } else {
        share[p][0] = static_cast<float>(a.counts[e]) * per_pair;
      }
    }
  }
  for (long base = static_cast<long>(blockIdx.x) * groups; base < a.T; base += step, t += step) {
    const bool any = on != 0 && lse != -INFINITY;      // else the token does not count, or has no finite logit
    const float level = any ? lse * to_z : 0.0f;
    float e[P][N], out[P][N], sums[2] = {0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int q = 0; q < N; ++q) {
        e[p][q] = any ? expf(v[p][q] - lse) : 0.0f;
        out[p][q] = more[p][q];
        sums[0] += e[p][q];
        sums[1] += share[p][q] * e[p][q];
      }
    if (base + step < a.T) fetch(t + step);
    // the sum of exp(z - lse) is 1 but for the rounding of lse, which dividing by it takes out of the probabilities
    const float total = lanes_sum(sums[0], a.lanes), scale = total == 0.0f ? 0.0f : 1.0f / total, mean = lanes_sum(sums[1], a.lanes) * scale;
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int c = (p * a.lanes + lane) * N;
#pragma unroll
      for (int q = 0; q < N; ++q) out[p][q] += e[p][q] * scale * ((share[p][q] - mean) * to_balance + level);
      if (t < a.T && c < a.E) store(out[p], a.dlogits + t * a.E + c);
    }
  }
}

// How the E columns of a row are dealt out: four pieces a lane where the row has as many
struct Split { int width, lanes, pieces; };
Split split_columns(int E) {
  Split s{E % 4 == 0 ? 4 : 1, 1, 1};
  const int pieces = E / s.width;
  while (s.lanes < 64 && s.lanes * 4 < pieces) s.lanes *= 2;
  while (s.lanes * s.pieces < pieces) s.pieces *= 2;
  return s;
}
int fwd_blocks(int T, int E) {
  const int rows = kFwdThreads / split_columns(E).lanes, n = T / rows + (T % rows != 0);
  return n < 1 ? 1 : n < kFwdBlocks ? n : kFwdBlocks;
}

int32_t check_balance(const char* who, int T, int E, int k) {
  MOE_REQUIRE(T >= 0 && E > 0 && k > 0, MOE_ERR_INVALID_ARG, "%s: need T >= 0, E > 0, k > 0 (T=%d E=%d k=%d)", who, T, E, k);
  MOE_REQUIRE(k <= E, MOE_ERR_INVALID_ARG, "%s: k=%d exceeds E=%d", who, k, E);
  MOE_REQUIRE(E <= kMaxExperts, MOE_ERR_UNSUPPORTED, "%s: E=%d above the built maximum %d", who, E, kMaxExperts);
  MOE_REQUIRE(k <= kMaxTopK, MOE_ERR_UNSUPPORTED, "%s: k=%d above the built maximum %d", who, k, kMaxTopK);
  MOE_REQUIRE(static_cast<int64_t>(T) * k <= INT32_MAX, MOE_ERR_UNSUPPORTED, "%s: T*k does not fit in int32", who);
  return MOE_OK;
}

template <class F> void with_split(const Split& s, F f) {
  using std::integral_constant;
  if (s.width == 4) {
    if (s.pieces == 1) f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    else if (s.pieces == 2) f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    else f(integral_constant<int, 4>{}, integral_constant<int, 4>{});
  } else {
    if (s.pieces <= 4) f(integral_constant<int, 1>{}, integral_constant<int, 4>{});
    else f(integral_constant<int, 1>{}, integral_constant<int, 16>{});
  }
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" size_t moe_balance_loss_fwd_workspace_bytes(int T, int E, int k) {
  (void)k;
  if (T < 0 || E <= 0 || E > kMaxExperts) return 0;
  const size_t blocks = fwd_blocks(T, E);
  return align_up(blocks * (2 * static_cast<size_t>(E) + 2) * 4, 16) + kHeadBytes;
}

extern "C" int32_t moe_balance_loss_fwd(const float* logits, const int32_t* topk_idx, const uint8_t* valid, int T, int E, int k, float* losses, int32_t* counts,
                                        float* importance, float* lse, void* ws, size_t ws_bytes, void* stream) {
  if (int32_t rc = check_balance("balance_loss_fwd", T, E, k)) return rc;
  MOE_REQUIRE(losses && counts && importance && (T == 0 || (logits && topk_idx && lse)), MOE_ERR_INVALID_ARG, "balance_loss_fwd: null pointer");
  MOE_REQUIRE(aligned16(logits) && aligned16(topk_idx) && aligned16(losses) && aligned16(counts) && aligned16(importance) && aligned16(lse), MOE_ERR_INVALID_ARG,
              "balance_loss_fwd: tensors must be 16-byte aligned");
  const size_t need = moe_balance_loss_fwd_workspace_bytes(T, E, k);
  MOE_REQUIRE(ws && ws_bytes >= need && aligned16(ws), MOE_ERR_WORKSPACE, "balance_loss_fwd: workspace null, misaligned or smaller than %zu bytes", need);
  const Split s = split_columns(E);
  const int blocks = fwd_blocks(T, E);
  FwdArgs a{logits, topk_idx, valid, losses, importance, lse, counts, T, E, k, s.lanes, divisor(k), nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
  a.joined = static_cast<uint32_t*>(ws);
  a.loss_of = reinterpret_cast<double*>(static_cast<char*>(ws) + 16);                 // of the join's workgroups
  static_assert(16 + kMaxExperts / kJoinLanes * sizeof(double) <= kHeadBytes);
  a.sum_of = reinterpret_cast<float*>(static_cast<char*>(ws) + kHeadBytes);
  a.count_of = reinterpret_cast<int32_t*>(a.sum_of + static_cast<size_t>(blocks) * E);
  a.z_of = reinterpret_cast<float*>(a.count_of + static_cast<size_t>(blocks) * E);
  a.n_of = reinterpret_cast<int32_t*>(a.z_of + blocks);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const size_t lds = (kFwdWaves + 1) * static_cast<size_t>(E) * 4;
  begin_call("moe_balance_loss_fwd", st);
  with_split(s, [&](auto n, auto p) {
    constexpr int N = decltype(n)::value, P = decltype(p)::value;
    if (blocks == 1) MOE_LAUNCH("balance_fwd", (balance_fwd_kernel<N, P, true>), dim3(1), dim3(kFwdThreads), lds, st, a);
    else MOE_LAUNCH("balance_fwd", (balance_fwd_kernel<N, P, false>), dim3(blocks), dim3(kFwdThreads), lds, st, a);
  });
  if (blocks > 1) {
    const int pieces = E / s.width;
    int lanes = 1;
    while (lanes < pieces && lanes < kJoinLanes) lanes *= 2;
    if (s.width == 4) MOE_LAUNCH("balance_join", balance_join_kernel<4>, dim3(ceil_div(pieces, lanes)), dim3(kJoinThreads), 0, st, a, blocks, lanes);
    else MOE_LAUNCH("balance_join", balance_join_kernel<1>, dim3(ceil_div(pieces, lanes)), dim3(kJoinThreads), 0, st, a, blocks, lanes);
  }
  return end_call();
}

extern "C" int32_t moe_balance_loss_bwd(const float* logits, const int32_t* counts, const float* lse, const uint8_t* valid, int T, int E, int k, float balance, float z,
                                        const float* dlosses, const float* add, float* dlogits, void* stream) {
  if (int32_t rc = check_balance("balance_loss_bwd", T, E, k)) return rc;
  if (T == 0) return MOE_OK;
  MOE_REQUIRE(logits && counts && lse && dlogits, MOE_ERR_INVALID_ARG, "balance_loss_bwd: null pointer");
  MOE_REQUIRE(aligned16(logits) && aligned16(counts) && aligned16(lse) && aligned16(dlosses) && aligned16(add) && aligned16(dlogits), MOE_ERR_INVALID_ARG,
              "balance_loss_bwd: tensors must be 16-byte aligned");
  const Split s = split_columns(E);
  BwdArgs a{logits, counts, lse, valid, dlosses, add, dlogits, T, E, k, s.lanes, balance, z};
  const int rows = kBwdThreads / s.lanes, blocks = T / rows + (T % rows != 0);
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_balance_loss_bwd", st);
  with_split(s, [&](auto n, auto p) {
    constexpr int N = decltype(n)::value, P = decltype(p)::value;
    MOE_LAUNCH("balance_bwd", (balance_bwd_kernel<N, P>), dim3(blocks < kBwdBlocks ? blocks : kBwdBlocks), dim3(kBwdThreads), 0, st, a);
  });
  return end_call();
}
