// A lane's share of a row: 16 consecutive bytes (rope.hip, norm.hip, balance.hip), and what rows in lanes need.
#pragma once
#include "moe_common.h"
#include "row_plan.h"

namespace moe {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// N consecutive elements of a row as they lie in memory: 16 bytes (32 in rope.hip's fp32 heads of more than 64 pieces of 16).
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
  __device__ __forceinline__ void hide() { asm volatile("" : "+v"(w)); }   // what was computed from it before is not kept for what follows
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

// ---- short rows side by side in a wave -----------------------------------------------------------------------
// f folded over the `lanes` (a power of two) consecutive lanes that share a row, in registers; all of them get the same bits.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <class F> __device__ __forceinline__ float lanes_fold(float v, int lanes, F f) {
  if (lanes > 1) v = f(v, dpp<0xB1>(v));               // quad_perm [1, 0, 3, 2]
  if (lanes > 2) v = f(v, dpp<0x4E>(v));               // quad_perm [2, 3, 0, 1]
  if (lanes > 4) v = f(v, dpp<0x141>(v));              // row_half_mirror
  if (lanes > 8) v = f(v, dpp<0x140>(v));              // row_mirror
  if (lanes > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if (lanes > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) { return lanes_fold(v, lanes, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float lanes_max(float v, int lanes) { return lanes_fold(v, lanes, [](float a, float b) { return fmaxf(a, b); }); }

}  // namespace moe
