// Codes of the 8-bit cache: bf16 <-> 8-bit floating point with a power-of-two scale.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sa.h"

namespace sa {

// log2 of the scale of values whose largest magnitude has the bf16 bits m (finite): least e >= -100 with
// m <= 2^e * largest, largest = 1.75 * 2^8 (e4m3) or 1.75 * 2^15 (e5m2); 0 for m = 0.  The lower end keeps every
// code * 2^e a normal bf16 value (the least is 2^-116).
template <int TYPE>
__device__ inline int scale_exponent(uint32_t m) {
  const int top = TYPE == SA_CACHE_E4M3 ? 8 : 15;
  const int e = (int)(m >> 7) - 127 - top + ((m & 0x7Fu) > 0x60u ? 1 : 0);
  return m == 0u ? 0 : max(e, -100);
}

// Four bf16 values (two words) times `inverse`, rounded to codes (ties to even).
template <int TYPE>
__device__ inline uint32_t encode4(uint32_t lo, uint32_t hi, float inverse) {
  const float f0 = __uint_as_float(lo << 16) * inverse, f1 = __uint_as_float(lo & 0xFFFF0000u) * inverse;
  const float f2 = __uint_as_float(hi << 16) * inverse, f3 = __uint_as_float(hi & 0xFFFF0000u) * inverse;
  int r = 0;
  if constexpr (TYPE == SA_CACHE_E4M3) {
    r = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, r, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, r, true);
  } else {
    r = __builtin_amdgcn_cvt_pk_bf8_f32(f0, f1, r, false);
    r = __builtin_amdgcn_cvt_pk_bf8_f32(f2, f3, r, true);
  }
  return (uint32_t)r;
}

typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
typedef float f32_pair __attribute__((ext_vector_type(2)));

// Codes 2 HALF, 2 HALF + 1 of a word times `scale` (a power of two) as bf16: exact.
template <int TYPE, bool HALF>
__device__ inline uint32_t decode2(uint32_t w, float scale) {
  bf16_pair r;
  if constexpr (TYPE == SA_CACHE_E4M3) r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HALF);
  else r = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, HALF);
  return __builtin_bit_cast(uint32_t, r);
}

// Codes 2 HALF, 2 HALF + 1 of a word as fp32.
template <int TYPE, bool HALF>
__device__ inline f32_pair decode2f(uint32_t w) {
  if constexpr (TYPE == SA_CACHE_E4M3) return __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HALF);
  else return __builtin_amdgcn_cvt_pk_f32_bf8((int)w, HALF);
}

// Bit 7 of every byte of a word of codes that is an infinity or NaN; and the word with 0 in their place.
template <int TYPE>
__device__ inline uint32_t nonfinite_codes(uint32_t w) {
  return ((w & 0x7F7F7F7Fu) + (TYPE == SA_CACHE_E4M3 ? 0x01010101u : 0x04040404u)) & 0x80808080u;
}
template <int TYPE>
__device__ inline uint32_t finite_codes(uint32_t w) {
  const uint32_t bad = nonfinite_codes<TYPE>(w);
  return w & ~((bad << 1) - (bad >> 7));
}

}  // namespace sa
