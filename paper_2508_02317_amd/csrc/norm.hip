// The norm in front of each half of a block, forward and backward: layer norm, or rms norm (no mean taken off), of rows of D elements.
//
//     h = x (+ residual),  m = mean(h) (rms: 0),  r = 1 / sqrt(mean((h - m)^2) + eps),  xh = (h - m) r,  y = xh w + b
//     dx = r (g - mean(g) - xh mean(g xh)) (+ add),  g = dy w  (rms: without mean(g));   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Bound by HBM: every tensor is read or written once.  A row is held in registers by a group of lanes from its one read to its writes: up to 64 lanes of a
// wave (several short rows side by side), or whole waves that exchange their sums through LDS.  A lane owns the same columns of all rows that its group
// walks, so weights are read once, and the sums over rows that the weights' gradients are stay in its registers until the end; workgroups leave
// them in the workspace and a second launch adds them in a fixed order.
// h is rounded to the element type before the norm is taken of it: it is what the next layer adds to and what the backward pass reads.
#include "moe_common.h"
#include "pieces.h"

namespace moe {

namespace {

constexpr int kMaxDim = 16384;
constexpr int kMaxPieces = 4;                          // 16-byte pieces of a row that one lane holds
constexpr int kFwdThreads = 256, kBwdThreads = 512;    // at least; a row of more waves has a workgroup of them
constexpr int kFwdBlocks = 2048, kBwdBlocks = 256;     // at most
constexpr int kJoinColumns = 64, kJoinThreads = 1024;

struct Rows {                                          // [T, H, D] with any strides of tokens and heads
  void* p;
  int64_t st, sh;
};
struct NormArgs {
  Rows x, residual, sum, y;                            // forward; residual and sum may be null
  Rows dy, add, dx;                                    // backward; x too
  const void *weight, *bias;
  float *mean, *rstd;                                  // written by the forward pass, read by the backward
  float* partial;                                      // [workgroups][D] of dw, then of db
  int rows, heads, dim, weight_bf16, lanes, waves, want_dw, want_db;
  Divisor per_token;
  float eps, per_dim;                                  // 1 / D
};

template <class E> __device__ __forceinline__ E* at(const Rows& r, uint32_t t, uint32_t h) { return static_cast<E*>(r.p) + t * r.st + h * r.sh; }

// N consecutive weights as floats
template <int N> __device__ __forceinline__ void weights(float (&w)[N], const void* p, int bf16, int column) {
  if (bf16) {
    const uint16_t* src = static_cast<const uint16_t*>(p) + column;
#pragma unroll
    for (int q = 0; q < N; ++q) w[q] = bf16_to_f32(src[q]);
  } else {
    const f32x4* src = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + column);
#pragma unroll
    for (int q = 0; q < N; ++q) w[q] = src[q / 4][q % 4];
  }
}

// Where a lane stands: its group among the workgroup's, its place in the group, the lanes of a group.
struct Place {
  int group, lane, size, groups, wave;
  __device__ __forceinline__ Place(int lanes, int waves) {
    const int l = static_cast<int>(threadIdx.x) & 63;
    wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) >> 6);
    const int in_block = static_cast<int>(blockDim.x) >> 6;
    if (waves == 1) {
      const int abreast = 64 / lanes;
      group = wave * abreast + l / lanes; lane = l & (lanes - 1); size = lanes; groups = in_block * abreast;
    } else {
      group = wave / waves; lane = wave % waves * 64 + l; size = 64 * waves; groups = in_block / waves;
    }
  }
};

// The sums of K values over a group.  Where it is several waves: one barrier, two buffers in turn (a wave that writes the one it wrote two calls
// ago has passed the barrier between, which all waves reach after they have read it).  Called by all of the workgroup alike.
template <int K> struct Sums {
  float buf[2][16][K];
  __device__ __forceinline__ void operator()(float (&v)[K], int lanes, int waves, int wave, int& turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum(v[k], lanes);
    if (waves > 1) {
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) buf[turn][wave][k] = v[k];
      }
      __syncthreads();
      const int first = wave / waves * waves;
#pragma unroll
      for (int k = 0; k < K; ++k) v[k] = 0.0f;
      for (int i = 0; i < waves; ++i) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += buf[turn][first + i][k];
      }
      turn ^= 1;
    }
  }
};

// P pieces of N elements a lane, U rows at once
template <class E, int N, int P, int U, bool LAYER>
__global__ __launch_bounds__(1024) void norm_fwd_kernel(NormArgs a) {
  __shared__ Sums<U> sums;
  const Place me(a.lanes, a.waves);
  int turn = 0;
  float w[P][N], b[P][N];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int column = (p * me.size + me.lane) * N;
#pragma unroll
    for (int q = 0; q < N; ++q) { w[p][q] = 1.0f; b[p][q] = 0.0f; }
    if (column < a.dim && a.weight) weights(w[p], a.weight, a.weight_bf16, column);
    if (column < a.dim && a.bias) weights(b[p], a.bias, a.weight_bf16, column);
  }
  const int step = me.groups * U;
  for (long base = static_cast<long>(blockIdx.x) * step; base < a.rows; base += static_cast<long>(gridDim.x) * step) {
    Piece<E, N> x[U][P], res[U][P];
    uint32_t t[U], h[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long row = base + u * me.groups + me.group;
      there[u] = row < a.rows;
      t[u] = there[u] ? divide(static_cast<uint32_t>(row), a.per_token) : 0;
      h[u] = there[u] ? static_cast<uint32_t>(row) - t[u] * a.heads : 0;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        const float zero[N] = {};
        x[u][p].set(zero);
        res[u][p].set(zero);
        if (there[u] && column < a.dim) {
          x[u][p].load(at<const E>(a.x, t[u], h[u]) + column);
          if (a.residual.p) res[u][p].load(at<const E>(a.residual, t[u], h[u]) + column);
        }
      }
    }
    float v[U][P][N], total[U], mean[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      total[u] = 0.0f;
      mean[u] = 0.0f;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        x[u][p].get(v[u][p]);
        if (a.residual.p) {
          float r[N];
          res[u][p].get(r);
#pragma unroll
          for (int q = 0; q < N; ++q) v[u][p][q] += r[q];
          x[u][p].set(v[u][p]);
          x[u][p].get(v[u][p]);
          if (there[u] && column < a.dim) x[u][p].store(at<E>(a.sum, t[u], h[u]) + column);
        }
#pragma unroll
        for (int q = 0; q < N; ++q) total[u] += LAYER ? v[u][p][q] : v[u][p][q] * v[u][p][q];
      }
    }
    sums(total, a.lanes, a.waves, me.wave, turn);
    if (LAYER) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        mean[u] = total[u] * a.per_dim;
        total[u] = 0.0f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if ((p * me.size + me.lane) * N < a.dim) {   // places that no column has stay out of the second sum
#pragma unroll
            for (int q = 0; q < N; ++q) {
              v[u][p][q] -= mean[u];
              total[u] += v[u][p][q] * v[u][p][q];
            }
          }
        }
      }
      sums(total, a.lanes, a.waves, me.wave, turn);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!there[u]) continue;
      const float rstd = 1.0f / sqrtf(total[u] * a.per_dim + a.eps);
      if (me.lane == 0) {
        const long row = base + u * me.groups + me.group;
        if (a.rstd) a.rstd[row] = rstd;
        if (LAYER && a.mean) a.mean[row] = mean[u];
      }
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        if (column >= a.dim) continue;
        float y[N];
#pragma unroll
        for (int q = 0; q < N; ++q) y[q] = v[u][p][q] * rstd * w[p][q] + b[p][q];
        Piece<E, N> o;
        o.set(y);
        o.store(at<E>(a.y, t[u], h[u]) + column);
      }
    }
  }
}

template <class E, int N, int P, int U, bool LAYER>
__global__ __launch_bounds__(sizeof(E) == 4 ? 1024 : 512) void norm_bwd_kernel(NormArgs a) {
  constexpr int K = LAYER ? 2 : 1;
  __shared__ Sums<U * K> sums;
  extern __shared__ __align__(16) float columns[];     // [half of the waves, or sets of them][D] of dw, then of db: 32 KiB at most
  const Place me(a.lanes, a.waves);
  int turn = 0;
  float w[P][N], dw[P][N], db[P][N];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int column = (p * me.size + me.lane) * N;
#pragma unroll
    for (int q = 0; q < N; ++q) { w[p][q] = 1.0f; dw[p][q] = 0.0f; db[p][q] = 0.0f; }
    if (column < a.dim && a.weight) weights(w[p], a.weight, a.weight_bf16, column);
  }
  const int step = me.groups * U;
  for (long base = static_cast<long>(blockIdx.x) * step; base < a.rows; base += static_cast<long>(gridDim.x) * step) {
    Piece<E, N> x[U][P], dy[U][P], add[U][P];
    uint32_t t[U], h[U];
    bool there[U];
    float mean[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long row = base + u * me.groups + me.group;
      there[u] = row < a.rows;
      t[u] = there[u] ? divide(static_cast<uint32_t>(row), a.per_token) : 0;
      h[u] = there[u] ? static_cast<uint32_t>(row) - t[u] * a.heads : 0;
      rstd[u] = there[u] ? a.rstd[row] : 0.0f;
      mean[u] = LAYER && there[u] ? a.mean[row] : 0.0f;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        const float zero[N] = {};
        x[u][p].set(zero);
        dy[u][p].set(zero);
        add[u][p].set(zero);
        if (there[u] && column < a.dim) {
          x[u][p].load(at<const E>(a.x, t[u], h[u]) + column);
          dy[u][p].load(at<const E>(a.dy, t[u], h[u]) + column);
          if (a.add.p) add[u][p].load(at<const E>(a.add, t[u], h[u]) + column);
        }
      }
    }
    float xh[U][P][N], g[U][P][N], total[U * K];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int k = 0; k < K; ++k) total[u * K + k] = 0.0f;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        float d[N];
        x[u][p].get(xh[u][p]);
        dy[u][p].get(d);
#pragma unroll
        for (int q = 0; q < N; ++q) {
          xh[u][p][q] = (xh[u][p][q] - mean[u]) * rstd[u];
          dw[p][q] += d[q] * xh[u][p][q];
          db[p][q] += d[q];
          g[u][p][q] = d[q] * w[p][q];
          total[u * K] += g[u][p][q] * xh[u][p][q];
          if (LAYER) total[u * K + K - 1] += g[u][p][q];
        }
      }
    }
    sums(total, a.lanes, a.waves, me.wave, turn);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!there[u]) continue;
      const float along = total[u * K] * a.per_dim, level = LAYER ? total[u * K + K - 1] * a.per_dim : 0.0f;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        if (column >= a.dim) continue;
        float o[N], more[N];
        add[u][p].get(more);
#pragma unroll
        for (int q = 0; q < N; ++q) o[q] = (g[u][p][q] - level - xh[u][p][q] * along) * rstd[u] + more[q];
        Piece<E, N> out;
        out.set(o);
        out.store(at<E>(a.dx, t[u], h[u]) + column);
      }
    }
  }
  // the sums over the workgroup's rows: over the groups of a wave in registers, then over the waves (or sets of them) in the order of their numbers
  const int units = (static_cast<int>(blockDim.x) >> 6) / a.waves, unit = me.wave / a.waves;
  const bool owner = a.waves > 1 || (static_cast<int>(threadIdx.x) & 63) < a.lanes;
  auto leave = [&](float (&acc)[P][N], float* dst) {
    for (int o = a.lanes; o < 64; o *= 2) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int q = 0; q < N; ++q) acc[p][q] += __shfl_xor(acc[p][q], o, 64);
    }
    // f(where a piece lies among the D, its four sums at a time)
    auto pieces = [&](bool who, auto f) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        if (who && owner && column < a.dim) {
#pragma unroll
          for (int q = 0; q < N; q += 4) f(column + q, f32x4{acc[p][q], acc[p][q + 1], acc[p][q + 2], acc[p][q + 3]});
        }
      }
    };
    auto quad = [](float* at) -> f32x4& { return *reinterpret_cast<f32x4*>(at); };
    if (units == 1) {
      pieces(true, [&](int c, f32x4 v) { quad(dst + c) = v; });
      return;
    }
    // the upper half of the units leaves its sums, the lower half adds its own, all threads add those
    const int half = units / 2;
    float* place = columns + (unit % half) * a.dim;
    pieces(unit >= half, [&](int c, f32x4 v) { quad(place + c) = v; });
    __syncthreads();
    pieces(unit < half, [&](int c, f32x4 v) { quad(place + c) += v; });
    __syncthreads();
    for (int c = 4 * threadIdx.x; c < a.dim; c += 4 * blockDim.x) {
      f32x4 v = quad(columns + c);
      for (int i = 1; i < half; ++i) v += quad(columns + i * a.dim + c);
      quad(dst + c) = v;
    }
    __syncthreads();
  };
  float* mine = a.partial + static_cast<long>(blockIdx.x) * a.dim;
  if (a.want_dw) leave(dw, mine);
  if (a.want_db) leave(db, mine + static_cast<long>(gridDim.x) * a.dim);
}

// [parts][D] -> [D] in the weights' type: a lane has four columns of every kJoinRuns-th part, then the runs are added, over a wave and over the waves.
__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const float* partial, int parts, int dim, void* dweight, void* dbias, int bf16) {
  constexpr int kQuads = kJoinColumns / 4, kRuns = kJoinThreads / kQuads, kWaves = kJoinThreads / 64;
  __shared__ float run[kWaves][kJoinColumns];
  const int c = 4 * (static_cast<int>(threadIdx.x) % kQuads), r = static_cast<int>(threadIdx.x) / kQuads, column = blockIdx.x * kJoinColumns + c;
  const float* src = partial + static_cast<long>(blockIdx.y) * parts * dim;
  void* dst = blockIdx.y ? dbias : dweight;
  if (!dst) return;
  f32x4 v = {};
  if (column < dim) {
#pragma unroll 4
    for (int i = r; i < parts; i += kRuns) v += *reinterpret_cast<const f32x4*>(src + static_cast<long>(i) * dim + column);
  }
#pragma unroll
  for (int o = kQuads; o < 64; o *= 2)
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += __shfl_xor(v[q], o, 64);
  if ((threadIdx.x & 63) < kQuads) *reinterpret_cast<f32x4*>(&run[threadIdx.x >> 6][c]) = v;
  __syncthreads();
  const int mine = blockIdx.x * kJoinColumns + threadIdx.x;
  if (threadIdx.x < kJoinColumns && mine < dim) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) sum += run[i][threadIdx.x];
    if (bf16) static_cast<bf16_t*>(dst)[mine] = f32_to_bf16(sum);
    else static_cast<float*>(dst)[mine] = sum;
  }
}

// How rows of D elements are dealt out to lanes.
struct Split { int lanes, waves, pieces; };
Split split_row(int dtype, int D) {
  const int pieces = D / (16 / elem_size(dtype));
  Split s{1, 1, 1};
  while (s.lanes < 64 && s.lanes < pieces) s.lanes *= 2;
  while (s.waves * 64 * kMaxPieces < pieces) s.waves *= 2;
  while (s.lanes * s.waves * s.pieces < pieces) s.pieces *= 2;
  return s;
}
int threads_of(const Split& s, int least) { return s.waves * 64 > least ? s.waves * 64 : least; }
int groups_of(const Split& s, int threads) { return s.waves > 1 ? threads / 64 / s.waves : threads / s.lanes; }
int blocks_of(int rows, const Split& s, int threads, int most) {
  const int step = groups_of(s, threads) * (kMaxPieces / s.pieces), n = rows / step + (rows % step != 0);
  return n < most ? n : most;
}

template <bool BACK, class E, int N, int P, bool LAYER> void launch_norm(const NormArgs& a, int blocks, int threads, hipStream_t st) {
  if constexpr (BACK)
    MOE_LAUNCH("norm_bwd", (norm_bwd_kernel<E, N, P, kMaxPieces / P, LAYER>), dim3(blocks), dim3(threads), (a.want_dw || a.want_db) && threads / 64 > a.waves ? threads / 64 / a.waves / 2 * a.dim * 4 : 0, st, a);
  else
    MOE_LAUNCH("norm_fwd", (norm_fwd_kernel<E, N, P, kMaxPieces / P, LAYER>), dim3(blocks), dim3(threads), 0, st, a);
}
template <bool BACK> void launch_norm(const NormArgs& a, const Split& s, int dtype, bool layer, int blocks, int threads, hipStream_t st) {
  auto typed = [&](auto e, auto n) {
    typedef decltype(e) E;
    constexpr int N = decltype(n)::value;
    if (layer) {
      if (s.pieces == 1) launch_norm<BACK, E, N, 1, true>(a, blocks, threads, st);
      else if (s.pieces == 2) launch_norm<BACK, E, N, 2, true>(a, blocks, threads, st);
      else launch_norm<BACK, E, N, 4, true>(a, blocks, threads, st);
    } else {
      if (s.pieces == 1) launch_norm<BACK, E, N, 1, false>(a, blocks, threads, st);
      else if (s.pieces == 2) launch_norm<BACK, E, N, 2, false>(a, blocks, threads, st);
      else launch_norm<BACK, E, N, 4, false>(a, blocks, threads, st);
    }
  };
  if (dtype == MOE_BF16) typed(bf16_t{}, std::integral_constant<int, 8>{});
  else typed(float{}, std::integral_constant<int, 4>{});
}

int32_t check_norm(const char* who, int dtype, int weight_dtype, int T, int H, int D) {
  MOE_REQUIRE(dtype == MOE_F32 || dtype == MOE_BF16, MOE_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
  MOE_REQUIRE(weight_dtype == MOE_F32 || weight_dtype == MOE_BF16, MOE_ERR_UNSUPPORTED, "%s: unknown dtype %d of the weights", who, weight_dtype);
  MOE_REQUIRE(T >= 0 && H > 0 && D > 0, MOE_ERR_INVALID_ARG, "%s: need T >= 0, H > 0 and D > 0 (T=%d H=%d D=%d)", who, T, H, D);
  MOE_REQUIRE(D % 8 == 0 && D <= kMaxDim, MOE_ERR_UNSUPPORTED, "%s: D=%d must be a multiple of 8 up to %d", who, D, kMaxDim);
  MOE_REQUIRE(static_cast<int64_t>(T) * H <= INT32_MAX, MOE_ERR_UNSUPPORTED, "%s: T*H does not fit in int32", who);
  return MOE_OK;
}
bool rows_ok(int dtype, const Rows& r) {
  const int n = 16 / elem_size(dtype);
  return aligned16(r.p) && r.st % n == 0 && r.sh % n == 0;
}
Rows rows(const void* p, int64_t st, int64_t sh) { return Rows{const_cast<void*>(p), st, sh}; }

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" int32_t moe_norm_fwd(const void* x, int64_t x_stride_t, int64_t x_stride_h, const void* residual, int64_t r_stride_t, int64_t r_stride_h, int dtype,
                                int T, int H, int D, int rms, const void* weight, const void* bias, int weight_dtype, float eps, void* sum, int64_t s_stride_t,
                                int64_t s_stride_h, void* y, int64_t y_stride_t, int64_t y_stride_h, float* mean, float* rstd, void* stream) {
  if (int32_t rc = check_norm("norm_fwd", dtype, weight_dtype, T, H, D)) return rc;
  MOE_REQUIRE(eps >= 0.0f && eps < INFINITY, MOE_ERR_INVALID_ARG, "norm_fwd: eps=%g must be a finite number of 0 or more", static_cast<double>(eps));
  MOE_REQUIRE((residual != nullptr) == (sum != nullptr), MOE_ERR_INVALID_ARG, "norm_fwd: residual and sum come together");
  if (T == 0) return MOE_OK;
  MOE_REQUIRE(x && y, MOE_ERR_INVALID_ARG, "norm_fwd: null pointer");
  NormArgs a{};
  a.x = rows(x, x_stride_t, x_stride_h); a.residual = rows(residual, r_stride_t, r_stride_h); a.sum = rows(sum, s_stride_t, s_stride_h); a.y = rows(y, y_stride_t, y_stride_h);
  MOE_REQUIRE(rows_ok(dtype, a.x) && rows_ok(dtype, a.y) && (!residual || (rows_ok(dtype, a.residual) && rows_ok(dtype, a.sum))) && aligned16(weight) && aligned16(bias),
              MOE_ERR_INVALID_ARG, "norm_fwd: tensors must be 16-byte aligned and strides multiples of 16 bytes");
  const Split s = split_row(dtype, D);
  const int threads = threads_of(s, kFwdThreads);
  a.weight = weight; a.bias = bias; a.weight_bf16 = weight_dtype == MOE_BF16; a.mean = mean; a.rstd = rstd; a.rows = T * H; a.heads = H; a.dim = D;
  a.lanes = s.lanes; a.waves = s.waves; a.per_token = divisor(H); a.eps = eps; a.per_dim = 1.0f / static_cast<float>(D);
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_norm_fwd", st);
  launch_norm<false>(a, s, dtype, !rms, blocks_of(a.rows, s, threads, kFwdBlocks), threads, st);
  return end_call();
}

extern "C" size_t moe_norm_bwd_workspace_bytes(int T, int H, int D) {
  if (T < 0 || H <= 0 || D <= 0) return 0;
  const int64_t rows = static_cast<int64_t>(T) * H;
  return align_up(static_cast<size_t>(rows < kBwdBlocks ? rows : kBwdBlocks) * D * 2 * sizeof(float), 256);
}

extern "C" int32_t moe_norm_bwd(const void* dy, int64_t dy_stride_t, int64_t dy_stride_h, const void* x, int64_t x_stride_t, int64_t x_stride_h, int dtype, int T,
                                int H, int D, const float* mean, const float* rstd, const void* weight, int weight_dtype, const void* add, int64_t add_stride_t,
                                int64_t add_stride_h, void* dx, int64_t dx_stride_t, int64_t dx_stride_h, void* dweight, void* dbias, void* ws, size_t ws_bytes,
                                void* stream) {
  if (int32_t rc = check_norm("norm_bwd", dtype, weight_dtype, T, H, D)) return rc;
  const bool wanted = dweight || dbias;
  if (T == 0 && !wanted) return MOE_OK;
  MOE_REQUIRE(T == 0 || (dy && x && rstd && dx), MOE_ERR_INVALID_ARG, "norm_bwd: null pointer");
  NormArgs a{};
  a.dy = rows(dy, dy_stride_t, dy_stride_h); a.x = rows(x, x_stride_t, x_stride_h); a.add = rows(add, add_stride_t, add_stride_h); a.dx = rows(dx, dx_stride_t, dx_stride_h);
  MOE_REQUIRE(rows_ok(dtype, a.dy) && rows_ok(dtype, a.x) && rows_ok(dtype, a.dx) && (!add || rows_ok(dtype, a.add)) && aligned16(weight) && aligned16(dweight) &&
              aligned16(dbias), MOE_ERR_INVALID_ARG, "norm_bwd: tensors must be 16-byte aligned and strides multiples of 16 bytes");
  const size_t need = moe_norm_bwd_workspace_bytes(T, H, D);
  MOE_REQUIRE(!wanted || (ws && ws_bytes >= need && aligned16(ws)), MOE_ERR_WORKSPACE, "norm_bwd: workspace null, misaligned or smaller than %zu bytes", need);
  const Split s = split_row(dtype, D);
  const int threads = threads_of(s, kBwdThreads), blocks = T ? blocks_of(T * H, s, threads, kBwdBlocks) : 0;
  a.weight = weight; a.weight_bf16 = weight_dtype == MOE_BF16; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.rows = T * H; a.heads = H; a.dim = D;
  a.lanes = s.lanes; a.waves = s.waves; a.per_token = divisor(H); a.per_dim = 1.0f / static_cast<float>(D);
  a.partial = wanted ? static_cast<float*>(ws) : nullptr; a.want_dw = dweight != nullptr; a.want_db = dbias != nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_norm_bwd", st);
  if (blocks) launch_norm<true>(a, s, dtype, mean != nullptr, blocks, threads, st);
  if (wanted)
    MOE_LAUNCH("norm_join", norm_join_kernel, dim3(ceil_div(D, kJoinColumns), dbias ? 2 : 1), dim3(kJoinThreads), 0, st, a.partial, blocks, D, dweight, dbias,
               weight_dtype == MOE_BF16);
  return end_call();
}
