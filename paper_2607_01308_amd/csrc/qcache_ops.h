// Device helpers of the 8-bit paged cache: e4m3 codes to and from the types that the
// kernels compute with. Codes to bf16 and to fp32 are exact (e4m3 has 4 exponent and 3
// mantissa bits); values to codes round to nearest even.
#pragma once

#include "qcache.h"

namespace cm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Two codes (the low or the high half of a word) as a bf16 pair.
template <bool HI>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}

// Two fp32 values as a bf16 pair, rounded to nearest even.
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi) {
  const f32x2v v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2v));
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) {
  return __uint_as_float(w & 0xFFFF0000u);
}

// Four fp32 values as four codes. |value| <= 448 or NaN.
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// max and sum of a value and that of the lane 16 or 32 away (exchanged within the
// vector registers, not through the LDS, whose queue they would wait for).
template <int BY>
__device__ __forceinline__ void lane_pair(float x, float& a, float& b) {
  const uint32_t u = __float_as_uint(x);
  if constexpr (BY == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
  } else {
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
  }
}
template <int BY>
__device__ __forceinline__ float lane_max(float x) {
  float a, b;
  lane_pair<BY>(x, a, b);
  return fmaxf(a, b);
}
template <int BY>
__device__ __forceinline__ float lane_sum(float x) {
  float a, b;
  lane_pair<BY>(x, a, b);
  return a + b;
}

// Bits of the least 2^e, e >= -120, with amax <= 448 * 2^e (448 = 1.75 * 2^8), from
// the bits of a finite amax >= 0.
__device__ __forceinline__ uint32_t scale_bits(uint32_t amax) {
  int e = (int)(amax >> 23) - 135 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = e < -120 ? -120 : e;
  return (uint32_t)(e + 127) << 23;
}

// 1 in each byte of a word of four codes that is NaN (0x7F, 0xFF): a byte of
// (w & 0x7F) + 1 reaches 0x80 only there.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) {
  return (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) >> 7;
}

}  // namespace cm
