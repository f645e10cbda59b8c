// Codes of the 4-bit cache: bf16 <-> groups of 32 codes e2m1 with one scale 2^e, kept as the byte e + 127 (255: NaN).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sa.h"

namespace sa {

constexpr int kGroup = 32;            // elements of a scale
constexpr int kRow4 = 64, kScales4 = 4;  // bytes of a row's codes, and of its scales
constexpr uint32_t kNanScale = 255u;

// log2 of the scale of a group whose largest magnitude has the bf16 bits m (finite): the least e in [-100, 125] with m < 7 * 2^e,
// 0 for m = 0.  Below 7 scales nothing rounds to a code behind 6, so no value is off by more than half a step; from 4 scales on 6 is the only code
// left, and a scale by "m <= 6 * 2^e" would take the next power of two, and twice the step for all, for one value between 6 and 7.  The lower
// end keeps code * 2^e a normal bf16 value, the upper one finite (6 * 2^125; values from 7 * 2^125 on become that).
__device__ inline int scale_exponent4(uint32_t m) {
  const int e = (int)(m >> 7) - 129 + ((m & 0x7Fu) >= 0x60u ? 1 : 0);  // 7 = 1.75 * 2^2
  return m == 0u ? 0 : min(max(e, -100), 125);
}

__device__ inline uint32_t max_halves(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Pair SLOT of a word of codes, from two bf16 values over `scale`, ties to even.
template <int SLOT>
__device__ inline uint32_t encode4_2(uint32_t old, uint32_t pair, float scale) {
  typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16_pair, pair), scale, SLOT);
}
__device__ inline uint32_t encode4_8(const uint4 x, float scale) {
  return encode4_2<3>(encode4_2<2>(encode4_2<1>(encode4_2<0>(0u, x.x, scale), x.y, scale), x.z, scale), x.w, scale);
}

// A scale byte as fp32.  255 becomes an infinity, which the conversions below take for NaN.
__device__ inline float scale4(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes 2 SLOT, 2 SLOT + 1 of a word times `scale`: exact.
template <int SLOT>
__device__ inline uint32_t decode4_2(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SLOT));
}
__device__ inline uint4 decode4_8(uint32_t w, float scale) {
  return make_uint4(decode4_2<0>(w, scale), decode4_2<1>(w, scale), decode4_2<2>(w, scale), decode4_2<3>(w, scale));
}

// Eight codes of a word times `scale` as fp32.
__device__ inline void decode4_8f(uint32_t w, float scale, float (&f)[8]) {
  typedef float f32_pair __attribute__((ext_vector_type(2)));
  const f32_pair a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const f32_pair c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  f[0] = a[0]; f[1] = a[1]; f[2] = b[0]; f[3] = b[1]; f[4] = c[0]; f[5] = c[1]; f[6] = d[0]; f[7] = d[1];
}

}  // namespace sa
