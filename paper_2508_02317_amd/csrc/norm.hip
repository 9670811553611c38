// The norm in front of each half of a block, forward and backward: layer norm, or rms norm (no mean taken off), of rows of D elements.
//
//     h = x (+ residual),  m = mean(h) (rms: 0),  r = 1 / sqrt(mean((h - m)^2) + eps),  xh = (h - m) r,  y = xh w + b
//     dx = r (g - mean(g) - xh mean(g xh)) (+ add),  g = dy w  (rms: without mean(g));   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Bound by HBM: every tensor is read or written once.  A row is held in registers by a group of lanes from its one read to its writes: up to 64 lanes of a
// wave (several short rows side by side), or whole waves that exchange their sums through LDS.  A lane owns the same columns of all rows that its group
// walks, so weights are read once, and the sums over rows that the weights' gradients are stay in its registers until the end; workgroups leave
// them in the workspace and a second launch adds them in a fixed order.
// h is rounded to the element type before the norm is taken of it: it is what the next layer adds to and what the backward pass reads.  Sums, statistics and
// the gradients' sums are fp32; y, dx, dw and db are rounded once.
// Measured in bf16 (a streaming copy moves 5.9 to 6.3 TB/s): 40960 rows of 2048 back, with an added gradient and the weight's, 671 MB, 109.5 us, 6.1 TB/s; forward with
// a residual 112 us, 6.0; 8192 rows forward 24.5, 5.5, back 27.8 (4.3 of it the second launch); 262144 heads of 128 back 38.7, 5.2 (the same); 16 rows 3.4 on the GPU.
#include "moe_common.h"
#include "pieces.h"

namespace moe {

namespace {

constexpr int kMaxDim = 16384;
// 16-byte pieces of a row that one lane holds; of shorter rows, several at once.  Back, a lane's registers hold weights, two sums and the next row beside a row: with
// four pieces 40960 rows of 2048 took 117 us, 110 with two, as layer norm with bias 189 (registers spilled), 111 with two.  Forward four are better: 8192 rows 24.5,
// 25.1 with two.  All in bf16; fp32, where two pieces are half the elements and registers, goes by the same numbers without measurements of its own.
constexpr int kFwdPieces = 4, kBwdPieces = 2;
constexpr int kFwdThreads = 256, kBwdThreads = 512, kMaxThreads = 1024;   // at least; a row of more waves has a workgroup of them
// at most: forward 40960 rows with residual 116.9 us with 2048, 112.2 with 4096, 111.1 with 8192, without residual 58.1, 56.4 and 61.4; back 256 leave the fewest
// sums (8192 rows 28.2, 31.8 with 512; 40960 rows 109.6 and 112.0)
constexpr int kFwdBlocks = 4096, kBwdBlocks = 256;
constexpr int kJoinColumns = 32, kJoinThreads = 512;    // 64 and 1024: 8192 rows back 28.0 us, 27.8 as it is

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

// P pieces of N elements a lane, U rows at once.  Loads are in straight-line code, at places that exist: one behind a branch is waited for where the paths meet.
template <class E, int N, int P, int U, bool LAYER, bool SUM>
__global__ __launch_bounds__(sizeof(E) == 2 ? kMaxThreads / 2 : kMaxThreads) void norm_fwd_kernel(NormArgs a) {
  __shared__ Sums<U> sums;
  const Place me(a.lanes, a.waves);
  int turn = 0;
  const long step = static_cast<long>(me.groups) * U, all = step * gridDim.x;
  Piece<E, N> x[U][P], res[U][P];
  uint32_t t[U], h[U];
  auto request = [&](long base) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t row = static_cast<uint32_t>(min(base + u * me.groups + me.group, a.rows - 1l));
      t[u] = divide(row, a.per_token);
      h[u] = row - t[u] * a.heads;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = min((p * me.size + me.lane) * N, a.dim - N);
        x[u][p].load(at<const E>(a.x, t[u], h[u]) + column);
        if constexpr (SUM) res[u][p].load(at<const E>(a.residual, t[u], h[u]) + column);
      }
    }
  };
  request(static_cast<long>(blockIdx.x) * step);
  float w[P][N], b[P][N];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int column = min((p * me.size + me.lane) * N, a.dim - N);
#pragma unroll
    for (int q = 0; q < N; ++q) { w[p][q] = 1.0f; b[p][q] = 0.0f; }
    if (a.weight) weights(w[p], a.weight, a.weight_bf16, column);
    if (a.bias) weights(b[p], a.bias, a.weight_bf16, column);
  }
  for (long base = static_cast<long>(blockIdx.x) * step; base < a.rows; base += all) {
    bool there[U];
    float v[U][P][N], total[U], mean[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      there[u] = base + u * me.groups + me.group < a.rows;
      total[u] = 0.0f;
      mean[u] = 0.0f;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        x[u][p].get(v[u][p]);
        if constexpr (SUM) {
          float r[N];
          res[u][p].get(r);
#pragma unroll
          for (int q = 0; q < N; ++q) v[u][p][q] += r[q];
          x[u][p].set(v[u][p]);
          x[u][p].get(v[u][p]);
          if (there[u] && column < a.dim) x[u][p].store(at<E>(a.sum, t[u], h[u]) + column);
        }
        if (column < a.dim) {
#pragma unroll
          for (int q = 0; q < N; ++q) total[u] += LAYER ? v[u][p][q] : v[u][p][q] * v[u][p][q];
        }
      }
    }
    uint32_t tt[U], hh[U];
#pragma unroll
    for (int u = 0; u < U; ++u) { tt[u] = t[u]; hh[u] = h[u]; }
    if (base + all < a.rows) request(base + all);
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
        o.store(at<E>(a.y, tt[u], hh[u]) + column);
      }
    }
  }
}

template <class E, int N, int P, int U, bool LAYER, bool WITH_DB, bool ADD, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_bwd_kernel(NormArgs a) {
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
  const long step = static_cast<long>(me.groups) * U, all = step * gridDim.x;
  // The next rows are requested when the present ones have been taken: loads in straight-line code, at places that exist, untouched until they are used (a
  // load behind a branch, or one that is masked at once, is waited for there).
  Piece<E, N> x[U][P], dy[U][P], add[U][P];
  uint32_t t[U], h[U];
  float mean_of[U], rstd_of[U];
  auto request = [&](long base) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t row = static_cast<uint32_t>(min(base + u * me.groups + me.group, a.rows - 1l));
      t[u] = divide(row, a.per_token);
      h[u] = row - t[u] * a.heads;
      rstd_of[u] = a.rstd[row];
      if constexpr (LAYER) mean_of[u] = a.mean[row];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = min((p * me.size + me.lane) * N, a.dim - N);
        x[u][p].load(at<const E>(a.x, t[u], h[u]) + column);
        dy[u][p].load(at<const E>(a.dy, t[u], h[u]) + column);
        if constexpr (ADD) add[u][p].load(at<const E>(a.add, t[u], h[u]) + column);
      }
    }
  };
  request(static_cast<long>(blockIdx.x) * step);
  for (long base = static_cast<long>(blockIdx.x) * step; base < a.rows; base += all) {
    float xh[U][P][N], g[U][P][N], total[U * K], rstd[U], mean[U];
    Piece<E, N> more[U][P];
    E* to[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      there[u] = base + u * me.groups + me.group < a.rows;
      to[u] = at<E>(a.dx, t[u], h[u]);
      rstd[u] = rstd_of[u];
      if constexpr (LAYER) mean[u] = mean_of[u];
#pragma unroll
      for (int k = 0; k < K; ++k) total[u * K + k] = 0.0f;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const bool real = there[u] && (p * me.size + me.lane) * N < a.dim;
        float d[N], v[N];
        x[u][p].get(v);
        dy[u][p].get(d);
        if constexpr (ADD) more[u][p] = add[u][p];
#pragma unroll
        for (int q = 0; q < N; ++q) {
          d[q] = real ? d[q] : 0.0f;
          xh[u][p][q] = real ? (LAYER ? v[q] - mean[u] : v[q]) * rstd[u] : 0.0f;
          g[u][p][q] = d[q] * w[p][q];
          dw[p][q] += d[q] * xh[u][p][q];
          if constexpr (WITH_DB) db[p][q] += d[q];
          total[u * K] += g[u][p][q] * xh[u][p][q];
          if (LAYER) total[u * K + K - 1] += g[u][p][q];
        }
      }
    }
    if (base + all < a.rows) request(base + all);
    sums(total, a.lanes, a.waves, me.wave, turn);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!there[u]) continue;
      const float along = total[u * K] * a.per_dim, level = LAYER ? total[u * K + K - 1] * a.per_dim : 0.0f;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const int column = (p * me.size + me.lane) * N;
        if (column >= a.dim) continue;
        float o[N];
        if constexpr (ADD) more[u][p].get(o);
#pragma unroll
        for (int q = 0; q < N; ++q) {
          const float own = (g[u][p][q] - level - xh[u][p][q] * along) * rstd[u];
          o[q] = ADD ? own + o[q] : own;
        }
        Piece<E, N> out;
        out.set(o);
        out.store(to[u] + column);
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

// [parts][D] -> [D] in the weights' type: a lane has four columns of every kRuns-th part, then the runs are added, over a wave and over the waves.
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
    if (bf16) static_cast<bf16_t*>(dst)[mine] = static_cast<bf16_t>(pack_bf16x2(sum, 0.0f));   // NaN stays NaN
    else static_cast<float*>(dst)[mine] = sum;
  }
}

RowSplit split_dim(int dtype, int D, int most) { return split_row(D / (16 / elem_size(dtype)), most); }

// f(element type, elements of a piece, pieces of a lane) of a split
template <class F> void with_split(const RowSplit& s, int dtype, F f) {
  using std::integral_constant;
  auto typed = [&](auto e, auto n) {
    if (s.pieces == 1) f(e, n, integral_constant<int, 1>{});
    else if (s.pieces == 2) f(e, n, integral_constant<int, 2>{});
    else f(e, n, integral_constant<int, 4>{});
  };
  if (dtype == MOE_BF16) typed(bf16_t{}, integral_constant<int, 8>{});
  else typed(float{}, integral_constant<int, 4>{});
}
void launch_fwd(const NormArgs& a, const RowSplit& s, int dtype, bool layer, int blocks, int threads, hipStream_t st) {
  with_split(s, dtype, [&](auto e, auto n, auto p) {
    auto launch = [&](auto kind, auto with_sum) {
      typedef decltype(e) E;
      constexpr int N = decltype(n)::value, P = decltype(p)::value, U = rows_at_once(P, kFwdPieces);
      MOE_LAUNCH("norm_fwd", (norm_fwd_kernel<E, N, P, U, decltype(kind)::value, decltype(with_sum)::value>), dim3(blocks), dim3(threads), 0, st, a);
    };
    auto kinds = [&](auto with_sum) { if (layer) launch(std::true_type{}, with_sum); else launch(std::false_type{}, with_sum); };
    if (a.residual.p) kinds(std::true_type{}); else kinds(std::false_type{});
  });
}
void launch_bwd(const NormArgs& a, const RowSplit& s, int dtype, bool layer, int blocks, int threads, hipStream_t st) {
  const int units = threads / 64 / a.waves;
  const size_t lds = (a.want_dw || a.want_db) && units > 1 ? static_cast<size_t>(units / 2) * a.dim * 4 : 0;
  with_split(s, dtype, [&](auto e, auto n, auto p) {
    auto launch = [&](auto kind, auto add) {
      typedef decltype(e) E;
      constexpr int N = decltype(n)::value, P = decltype(p)::value, U = rows_at_once(P, kBwdPieces), KIND = decltype(kind)::value;
      constexpr bool LAYER = KIND == 2, DB = KIND > 0, ADD = decltype(add)::value;
      if constexpr (P == kBwdPieces || (P > kBwdPieces && sizeof(E) == 4)) {
        if (threads > kBwdThreads) {                   // more than 8192 elements (bf16; 4096 in fp32): 128 registers a lane
          // Above 8192 elements all kinds but one spill, 12 to 42 registers in bf16, 22 to 120 in fp32.  8192 rows of 16384 in bf16: rms 141 us (none; 5.7 TB/s), with an
          // added gradient 210 (14 spilled; 5.1), layer norm with bias 185 (12), with both 363 (42; 3.0); 4096 rows in fp32 162, 426, 241 and 469 (22, 96, 49, 112)
          MOE_LAUNCH("norm_bwd", (norm_bwd_kernel<E, N, P, U, LAYER, DB, ADD, kMaxThreads>), dim3(blocks), dim3(threads), lds, st, a);
          return;
        }
      }
      if constexpr (P <= kBwdPieces) MOE_LAUNCH("norm_bwd", (norm_bwd_kernel<E, N, P, U, LAYER, DB, ADD, kBwdThreads>), dim3(blocks), dim3(threads), lds, st, a);
    };
    auto kinds = [&](auto add) {                       // a layer norm's bias has its sums beside the weight's, wanted or not
      if (layer) launch(std::integral_constant<int, 2>{}, add);
      else if (a.want_db) launch(std::integral_constant<int, 1>{}, add);
      else launch(std::integral_constant<int, 0>{}, add);
    };
    if (a.add.p) kinds(std::true_type{}); else kinds(std::false_type{});
  });
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
  const RowSplit s = split_dim(dtype, D, kFwdPieces);
  const int threads = threads_of(s, kFwdThreads);
  a.weight = weight; a.bias = bias; a.weight_bf16 = weight_dtype == MOE_BF16; a.mean = mean; a.rstd = rstd; a.rows = T * H; a.heads = H; a.dim = D;
  a.lanes = s.lanes; a.waves = s.waves; a.per_token = divisor(H); a.eps = eps; a.per_dim = 1.0f / static_cast<float>(D);
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_norm_fwd", st);
  launch_fwd(a, s, dtype, !rms, blocks_of(a.rows, s, threads, kFwdPieces, kFwdBlocks), threads, st);
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
  const RowSplit s = split_dim(dtype, D, kBwdPieces);
  const int threads = threads_of(s, kBwdThreads), blocks = T ? blocks_of(T * H, s, threads, kBwdPieces, kBwdBlocks) : 0;
  a.weight = weight; a.weight_bf16 = weight_dtype == MOE_BF16; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.rows = T * H; a.heads = H; a.dim = D;
  a.lanes = s.lanes; a.waves = s.waves; a.per_token = divisor(H); a.per_dim = 1.0f / static_cast<float>(D);
  a.partial = wanted ? static_cast<float*>(ws) : nullptr; a.want_dw = dweight != nullptr; a.want_db = dbias != nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  begin_call("moe_norm_bwd", st);
  if (blocks) launch_bwd(a, s, dtype, mean != nullptr, blocks, threads, st);
  if (wanted)
    MOE_LAUNCH("norm_join", norm_join_kernel, dim3(ceil_div(D, kJoinColumns), dbias ? 2 : 1), dim3(kJoinThreads), 0, st, a.partial, blocks, D, dweight, dbias,
               weight_dtype == MOE_BF16);
  return end_call();
}
