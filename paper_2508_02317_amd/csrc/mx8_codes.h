// MXFP8 blocks: 32 values with one power-of-two scale and E4M3 elements, on the device.
// (MX specification Sec. 6.3: shared exponent = floor(log2(max |v|)) - 8, elements rounded to nearest even and
// saturated at the largest E4M3 magnitude.)
#pragma once
#include <type_traits>
#include "moe_common.h"

namespace moe {

__device__ __forceinline__ float quad_max(float v) {
  auto dpp = [](float x, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0xB1>{}));   // quad_perm [1,0,3,2]
  v = fmaxf(v, dpp(v, std::integral_constant<int, 0x4E>{}));   // quad_perm [2,3,0,1]
  return v;
}
// E8M0 code of the scale of a block whose largest magnitude is amax (>= 0): biased exponent of amax minus 8, not below 0
__device__ __forceinline__ uint32_t mx_scale_code(float amax) {
  const uint32_t eb = __builtin_bit_cast(uint32_t, amax) >> 23;
  return eb > 8u ? eb - 8u : 0u;
}
// 1 / scale = 2^(127 - code), exact
__device__ __forceinline__ float mx_inverse_scale(uint32_t code) { return __builtin_bit_cast(float, (254u - code) << 23); }
// 2^(code - 127) for the scaled conversions, which look at its exponent alone: 0 stands for 2^-127, 255 for NaN
__device__ __forceinline__ float mx_scale(uint32_t code) { return __builtin_bit_cast(float, code << 23); }
// eight values -> eight E4M3 codes (the hardware conversion rounds to nearest even; it does not saturate)
__device__ __forceinline__ uint2 mx_encode8(const float (&v)[8], float inv) {
  float s[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) s[q] = __builtin_amdgcn_fmed3f(v[q] * inv, -448.0f, 448.0f);
  int w0 = __builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[1], 0, false);
  w0 = __builtin_amdgcn_cvt_pk_fp8_f32(s[2], s[3], w0, true);
  int w1 = __builtin_amdgcn_cvt_pk_fp8_f32(s[4], s[5], 0, false);
  w1 = __builtin_amdgcn_cvt_pk_fp8_f32(s[6], s[7], w1, true);
  return make_uint2(static_cast<uint32_t>(w0), static_cast<uint32_t>(w1));
}

__device__ __forceinline__ uint32_t mx_encode4(float a, float b, float c, float d, float inv) {
  auto s = [&](float v) { return __builtin_amdgcn_fmed3f(v * inv, -448.0f, 448.0f); };
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(s(a), s(b), 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(s(c), s(d), w, true));
}

}  // namespace moe
