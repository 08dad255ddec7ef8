// Rows held in 4 bits: blocks of 32 channels, each 32 codes of 4 bits (e2m1: a sign, and 0, 0.5, 1, 1.5, 2, 3, 4 or 6; the even channel in
// the low half of a byte) and a scale of 8 bits, 2^(scale - 127); 255 makes all of a block NaN.
//
// A block whose largest value is x has the smallest power of two that leaves x / 2^e below 7, which rounds to 6 at most: floor(log2 x) - 2,
// and one more from 1.75 * 2^floor(log2 x) on.  Division by 2^e is exact, so that a code is the value's one rounding, half way to even: off
// by half a step of e2m1, which is 2^e / 4 for values below 2 * 2^e, 2^e / 2 up to 4 * 2^e, and 2^e from there to 7 * 2^e.  Scales stay in
// 2 .. 252, where every value that they give is a normal number of bf16 and fp32: smaller blocks lose what lies below 2^-127, and the last
// eighth below 2^128 becomes 6 * 2^125.
#pragma once

#include "sl_common.h"

namespace sl {

#if defined(__HIPCC__)

typedef __bf16 fp4_bf16x2 __attribute__((ext_vector_type(2)));
typedef float fp4_f32x2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kNotFinite = 0x7f800000u;

// the scale of a block from the largest magnitude's bits
__device__ __forceinline__ uint32_t fp4_scale(uint32_t top) {
  if (top >= kNotFinite) return 255;
  const int e = (int)((top + 0x200000u) >> 23) - 2;
  return e < 2 ? 2 : e > 252 ? 252 : e;
}

// bits of 2^(scale - 127) as the conversions take them
__device__ __forceinline__ float fp4_power(uint32_t scale) { return __uint_as_float(scale << 23); }

// eight codes
__device__ __forceinline__ void fp4_to_f32(uint32_t w, uint32_t scale, float* f) {
  const float by = fp4_power(scale);
  const fp4_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 1);
  const fp4_f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 3);
  f[0] = a[0];
  f[1] = a[1];
  f[2] = b[0];
  f[3] = b[1];
  f[4] = c[0];
  f[5] = c[1];
  f[6] = d[0];
  f[7] = d[1];
}

// eight codes as 16 bytes of bf16
__device__ __forceinline__ uint4 fp4_to_bf16(uint32_t w, float by) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 3)));
}

// Eight codes as a row's elements: one piece of 16 bytes (bf16) or two (fp32).
template <typename T>
__device__ __forceinline__ void fp4_to_row8(uint32_t w, uint32_t scale, uint4* to) {
  if constexpr (sizeof(T) == 2) {
    to[0] = fp4_to_bf16(w, fp4_power(scale));
  } else {
    float f[8];
    fp4_to_f32(w, scale, f);
    to[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    to[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
  }
}

// a block's 32 codes as pieces of 16 bytes
template <typename T>
__device__ __forceinline__ void fp4_to_rows(const uint4& code, uint32_t scale, uint4* to) {
  constexpr int PER = sizeof(T) == 2 ? 1 : 2;
  fp4_to_row8<T>(code.x, scale, to);
  fp4_to_row8<T>(code.y, scale, to + PER);
  fp4_to_row8<T>(code.z, scale, to + 2 * PER);
  fp4_to_row8<T>(code.w, scale, to + 3 * PER);
}

// Eight elements (as fp4_to_row8 has them): the largest magnitude's bits, and their codes.
template <typename T>
__device__ __forceinline__ uint32_t largest_bits(const uint4* from) {
  uint32_t top = 0;
  const uint4 r = from[0];
  if constexpr (sizeof(T) == 2) {
    for (uint32_t w : {r.x, r.y, r.z, r.w}) top = max(max(top, w << 16 & 0x7fffffffu), w & 0x7fff0000u);
  } else {
    const uint4 s = from[1];
    for (uint32_t w : {r.x, r.y, r.z, r.w, s.x, s.y, s.z, s.w}) top = max(top, w & 0x7fffffffu);
  }
  return top;
}
template <typename T>
__device__ __forceinline__ uint32_t row8_to_fp4(const uint4* from, uint32_t scale) {
  if (scale == 255) return 0;
  const float by = fp4_power(scale);
  const uint4 r = from[0];
  uint32_t w = 0;
  if constexpr (sizeof(T) == 2) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(fp4_bf16x2, r.x), by, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(fp4_bf16x2, r.y), by, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(fp4_bf16x2, r.z), by, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(fp4_bf16x2, r.w), by, 3);
  } else {
    const uint4 s = from[1];
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(r.x), __uint_as_float(r.y), by, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(r.z), __uint_as_float(r.w), by, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(s.x), __uint_as_float(s.y), by, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(s.z), __uint_as_float(s.w), by, 3);
  }
  return w;
}

#endif  // __HIPCC__

}  // namespace sl
