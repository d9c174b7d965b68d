// Device-side helpers for the MX block formats (32 consecutive values and one
// power-of-two scale byte s, standing for 2^(s - 127); 255 marks a block with
// a NaN or an infinity): MX8 holds e4m3 values, MX4 e2m1 values.
#pragma once

#include "common.h"

namespace memfine {

typedef int32_t i32x8_t __attribute__((ext_vector_type(8)));

constexpr int kMxBlock = 32;
constexpr uint32_t kMxNan = 255;

// Scale byte of a block whose largest |x| has the bits `amax` (the maximum of
// the bit patterns as integers, so that a NaN wins): the smallest power of two
// for which the largest value of the format, kTop = 1.75 * 2^8 (e4m3) or 1.5 *
// 2^2 (e2m1), times it reaches amax, but at least 2^-127.
template <int kTopExp, uint32_t kTopMantissa> __device__ __forceinline__ uint32_t mx_scale(uint32_t amax) {
  const uint32_t ex = amax >> 23;
  if (ex == 255) return kMxNan;
  const int s = (int)ex - kTopExp + ((amax & 0x7fffffu) > kTopMantissa ? 1 : 0);
  return s > 0 ? (uint32_t)s : 0u;
}
__device__ __forceinline__ uint32_t mx8_scale(uint32_t amax) { return mx_scale<8, 0x600000u>(amax); }
__device__ __forceinline__ uint32_t mx4_scale(uint32_t amax) { return mx_scale<2, 0x400000u>(amax); }

// 2^(s - 127), also for s = 0 (a subnormal) and 255 (NaN).
__device__ __forceinline__ float mx_scale_value(uint32_t s) {
  return s == 0 ? __uint_as_float(0x400000u) : s == kMxNan ? __uint_as_float(0x7fc00000u)
                                                           : __uint_as_float(s << 23);
}
// 2^(127 - s), s <= 253: the factor that brings a block's values into the
// format's range (a power of two: the product rounds only where it is subnormal).
__device__ __forceinline__ float mx_inverse_scale(uint32_t s) {
  return s >= 254 ? __uint_as_float(0x400000u) : __uint_as_float((254u - s) << 23);
}

// Four floats of a block, already divided by its scale, as four e4m3 bytes
// (round to nearest, ties to even).
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return (uint32_t)v;
}

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The largest of the values of lanes l, l ^ 1 (and l ^ 2, ..., up to N lanes,
// N = 4 or 8, aligned), by DPP.
template <int kCtrl> __device__ __forceinline__ uint32_t umax_dpp(uint32_t v) {
  return umax(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xf, 0xf, false));
}
template <int N> __device__ __forceinline__ uint32_t lanes_umax(uint32_t v) {
  static_assert(N == 4 || N == 8, "4 or 8 lanes");
  v = umax_dpp<0xb1>(v);                          // quad_perm [1, 0, 3, 2]
  v = umax_dpp<0x4e>(v);                          // quad_perm [2, 3, 0, 1]
  if constexpr (N == 8) v = umax_dpp<0x141>(v);   // row_half_mirror
  return v;
}

}  // namespace memfine
