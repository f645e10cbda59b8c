// What the two kinds of causal attention over a cache share (8 bits: cache_attend.hip, 4 bits: cache4_attend.hip): the softmax step of a
// tile, the outputs of a row, and the join of the splits.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sa_internal.h"

namespace sa {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kMaxSplits = 256;

// Where a call's outputs go.
struct AttendOut {
  uint16_t *O;
  int64_t o_hs, o_rs;
  int g, Hkv, rows, S;  // query heads and query rows of a KV head, splits of the keys
  float *part;          // [Hkv * rows][S][128] unnormalised outputs of the splits
  float2 *ml;           // [Hkv * rows][S] their maxima and sums
};

__device__ inline float max_pair(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ inline float sum_pair(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ inline void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ inline float value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
// A read-only word at a wave-uniform address.
__device__ inline float uniform_load(const float *p, int i) {
  typedef const float __attribute__((address_space(4))) *const_f32p;
  return ((const_f32p)(uintptr_t)p)[i];
}

// A lane's half of a row, O^T accumulators: O / l in bf16, or the split's sums.
__device__ inline void put_row(const AttendOut &p, int kvh, int row, int head, int tok, int sp, int gg, float m, float l, const f32x16 (&o)[4]) {
  if (p.S > 1) {
    const size_t slot = ((size_t)kvh * p.rows + row) * p.S + sp;
    if (gg == 0) p.ml[slot] = make_float2(m, l);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *(float4 *)(p.part + slot * kHeadDim + 32 * db + 2 * r + 4 * gg) = make_float4(o[db][r], o[db][r + 1], o[db][r + 2], o[db][r + 3]);
  } else {
    const float inv = 1.f / l;
    uint16_t *out = p.O + (size_t)head * p.o_hs + (size_t)tok * p.o_rs;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const bf16x2 a = {(__bf16)(o[db][r] * inv), (__bf16)(o[db][r + 1] * inv)};
        const bf16x2 b = {(__bf16)(o[db][r + 2] * inv), (__bf16)(o[db][r + 3] * inv)};
        *(uint2 *)(out + 32 * db + 2 * r + 4 * gg) = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
      }
  }
}

// What the four waves of a workgroup have for the same 32 rows (lane q + 32 gg of each: half a row), joined through LDS that is free by
// the first barrier: O / l in bf16, or the split's sums.  so: [4][32][128].
__device__ inline void put_waves(const AttendOut &p, int kvh, int r0, int sp, float m_run, float l_run, const f32x16 (&oacc)[4], float *so,
                                 float (&s_m)[4][32], float (&s_l)[4][32]) {
  const int tid = threadIdx.x, q = tid & 31, gg = tid >> 5 & 1, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __syncthreads();
  if (gg == 0) { s_m[wave][q] = m_run; s_l[wave][q] = l_run; }
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; r += 4)
      *(float4 *)(so + (wave * 32 + q) * kHeadDim + ((32 * db + 2 * r + 4 * gg) ^ ((q & 7) << 2))) =
          make_float4(oacc[db][r], oacc[db][r + 1], oacc[db][r + 2], oacc[db][r + 3]);
  __syncthreads();
  const int mr = tid >> 3, d0 = (tid & 7) * 16;  // 16 outputs of a row each
  const int orow = r0 + mr;
  if (orow < p.rows) {
    float M = -INFINITY, L = 0.f, w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) M = fmaxf(M, s_m[k][mr]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[k] = s_m[k][mr] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[k][mr] - M);
      L += s_l[k][mr] * w[k];
    }
    const size_t slot = ((size_t)kvh * p.rows + orow) * p.S + sp;
    const float inv = p.S > 1 ? 1.f : 1.f / L;
    const int otok = orow / p.g;
    uint16_t *o = p.O + (size_t)(kvh * p.g + orow - otok * p.g) * p.o_hs + (size_t)otok * p.o_rs;
    if (p.S > 1 && d0 == 0) p.ml[slot] = make_float2(M, L);
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 x = *(const float4 *)(so + (k * 32 + mr) * kHeadDim + ((d0 + i) ^ ((mr & 7) << 2)));
        a.x = __builtin_fmaf(x.x, w[k], a.x); a.y = __builtin_fmaf(x.y, w[k], a.y);
        a.z = __builtin_fmaf(x.z, w[k], a.z); a.w = __builtin_fmaf(x.w, w[k], a.w);
      }
      if (p.S > 1) {
        *(float4 *)(p.part + slot * kHeadDim + d0 + i) = a;
      } else {
        const bf16x2 u = {(__bf16)(a.x * inv), (__bf16)(a.y * inv)}, v = {(__bf16)(a.z * inv), (__bf16)(a.w * inv)};
        *(uint2 *)(o + d0 + i) = make_uint2(__builtin_bit_cast(uint32_t, u), __builtin_bit_cast(uint32_t, v));
      }
    }
  }
}

#define SA_VTR(tile, db, key0) \
  __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((const char *)(tile) + ((vbase ^ (unsigned)((db) << 6)) + (key0) * 256)))

// A tile's scores (lane = row, accumulator r of half hf <-> key 32hf + 8(r/4) + 4gg + r%4 of HF * 32) into a row's running
// softmax and its outputs.  masked: keys from place lim + 1 (less 4gg) on are not seen.
// PARTS: the matrix instruction takes probabilities in bf16.  1: rounded to it, 2^-8 of each, which adds to an output as much error as
// its own rounding does (0.0023 of the outputs' scale, rounding alone 0.0017).  2: a leading part and the rest, 2^-15, by twice
// the products: 0.0017.  launch_cache_attend says which.
template <int PARTS, int HF>
__device__ inline void absorb_tile(f32x16 (&sacc)[HF], bool masked, int lim, const uint16_t *Vt, unsigned vbase, float c,
                                   float &m_run, f32x4 (&lacc)[2], f32x16 (&oacc)[4]) {
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  if (masked) {
#pragma unroll
    for (int hf = 0; hf < HF; ++hf)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (32 * hf + 8 * (r / 4) + r % 4 > lim) sacc[hf][r] = -INFINITY;
  }
  __builtin_amdgcn_s_setprio(0);
  float tmax = -INFINITY;
#pragma unroll
  for (int hf = 0; hf < HF; ++hf)
#pragma unroll
    for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, sacc[hf][r]);
  // The reference moves only when some row's maximum grew by more than 2^8: until then probabilities may exceed 1
  // (by at most 256x), which fp32 sums and bf16 P hold easily, and the 64 accumulators are not rescaled.
  if (__any(__builtin_fmaf(tmax, c, -m_run) > 8.f)) {
    const float m_new = fmaxf(m_run, max_pair(tmax) * c);
    const float alpha = __builtin_amdgcn_exp2f(m_run - ((m_new == -INFINITY) ? 0.f : m_new));
    m_run = m_new;
    lacc[0] *= alpha;
    lacc[1] *= alpha;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
  }
  const float m_ref = (m_run == -INFINITY) ? 0.f : m_run;
  // probabilities, a pair at a time, beside the products: see the sparse prefill for the order
  auto soft2 = [&](int g, int j) {
#pragma unroll
    for (int e = 2 * j; e < 2 * j + 2; ++e)
      sacc[g >> 1][8 * (g & 1) + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[g >> 1][8 * (g & 1) + e], c, -m_ref));
  };
  u32x4 pbuf[2][PARTS];
  auto cvt2 = [&](int g, int j) {
    const float a = sacc[g >> 1][8 * (g & 1) + 2 * j], b = sacc[g >> 1][8 * (g & 1) + 2 * j + 1];
    if constexpr (PARTS == 1) {
      const bf16x2 pr = {(__bf16)a, (__bf16)b};
      pbuf[g & 1][0][j] = __builtin_bit_cast(uint32_t, pr);
    } else {
      // The leading part is cut, not rounded, and the rest taken from p (1 + 2^-20), which the normaliser sees too: neither
      // part is negative, nor 0 or subnormal before p is below 2^-106, so that an infinite V stays infinite.
      const uint32_t wa = __float_as_uint(a), wb = __float_as_uint(b);
      const bf16x2 rest = {(__bf16)__builtin_fmaf(a, 1.f + 0x1p-20f, -__uint_as_float(wa & 0xFFFF0000u)),
                           (__bf16)__builtin_fmaf(b, 1.f + 0x1p-20f, -__uint_as_float(wb & 0xFFFF0000u))};
      pbuf[g & 1][0][j] = __builtin_amdgcn_perm(wb, wa, 0x07060302u);
      pbuf[g & 1][1][j] = __builtin_bit_cast(uint32_t, rest);
    }
  };
  // The normaliser sums the probabilities as multiplied, so that a row stays a convex combination of its V rows;
  // 4x4x4 products with ones do it on the matrix pipe.
  const s16x4 ones4 = {0x3f80, 0x3f80, 0x3f80, 0x3f80};
  s16x4 vlo[4], vhi[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) soft2(0, j);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    vlo[i] = SA_VTR(Vt, i & 3, 0);
    vhi[i] = SA_VTR(Vt, i & 3, 8);
  }
#pragma unroll
  for (int j = 0; j < 3; ++j) cvt2(0, j);
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int i = 0; i < 8 * HF; ++i) {
    const int g = i >> 2, db = i & 3;
    if (db == 0) {
      cvt2(g, 3);
#pragma unroll
      for (int x = 0; x < PARTS; ++x) asm("" : "+v"(pbuf[g & 1][x]));
    }
    const s16x8 av = __builtin_shufflevector(vlo[i & 3], vhi[i & 3], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
    for (int x = 0; x < PARTS; ++x) {
      const bf16x8 pb = __builtin_bit_cast(bf16x8, pbuf[g & 1][x]);
      oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, av), pb, oacc[db], 0, 0, 0);
      const s16x8 ps = __builtin_bit_cast(s16x8, pb);
      if (db == 0)
        lacc[0] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones4, __builtin_shufflevector(ps, ps, 0, 1, 2, 3), lacc[0], 0, 0, 0);
      if (db == 3)
        lacc[1] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones4, __builtin_shufflevector(ps, ps, 4, 5, 6, 7), lacc[1], 0, 0, 0);
    }
    if (i + 4 < 8 * HF) {
      vlo[i & 3] = SA_VTR(Vt, (i + 4) & 3, 16 * ((i + 4) >> 2));
      vhi[i & 3] = SA_VTR(Vt, (i + 4) & 3, 16 * ((i + 4) >> 2) + 8);
    }
    if (g + 1 < 2 * HF) {
      soft2(g + 1, db);
      if (db > 0) cvt2(g + 1, db - 1);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The splits of a row joined: WAVES waves per row, the reads of IN splits of a lane in flight at once.  1 wave: two outputs a lane;
// 4: half a wave a split, four outputs a lane.  The bound is the launch and one round trip to memory, since the partial rows come
// from other XCDs.  Hence (4, 16) beyond 32 splits, 128 of them in flight (against 32: 5 tokens of 8 heads at 10K keys, 81 splits,
// 11.3 -> 10.2 us, one token at 30K, 235 splits, 14.6 -> 11.6), and (4, 4) up to 32, where there may be thousands of rows and
// its registers would keep waves away (100 tokens of 32 heads at 10K keys, 16 splits, 33.8 us instead of 36.0).
// (The workgroup of a KV head that arrives last could join in the first launch: 0.4 to 5 us slower from 300 to 8000 keys,
// since it alone reads what this launch spreads.)
template <int WAVES, int IN>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendOut p) {
  constexpr int kSide = WAVES == 1 ? 1 : 2;               // splits that a wave reads side by side
  constexpr int kPer = WAVES == 1 ? 1 : kMaxSplits / 64;  // splits whose weight a lane takes
  constexpr int W = 2 * kSide, kLanes = kHeadDim / W;
  typedef float vec __attribute__((ext_vector_type(W)));
  typedef __bf16 bvec __attribute__((ext_vector_type(W)));
  __shared__ vec sums[kThreads / 64][kLanes];
  __shared__ float weights[kThreads / 64][64 * kPer];
  const int lane = threadIdx.x & 63, side = lane / kLanes, ln = lane % kLanes;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), k0 = wave % WAVES;
  const int all = p.Hkv * p.rows, at = min((int)blockIdx.x * (kThreads / 64 / WAVES) + wave / WAVES, all - 1);  // KV head, row
  float2 ml[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) ml[i] = lane + 64 * i < p.S ? p.ml[(size_t)at * p.S + lane + 64 * i] : make_float2(-INFINITY, 0.f);
  const float *src = p.part + (size_t)at * p.S * kHeadDim + W * ln;
  vec o = {}, x[IN];
  float L = 0.f;
  for (int s0 = kSide * k0; s0 < p.S; s0 += kSide * WAVES * IN) {
#pragma unroll
    for (int i = 0; i < IN; ++i) {
      const int s = s0 + kSide * WAVES * i;
      if (s < p.S) x[i] = *(const vec *)(src + (size_t)min(s + side, p.S - 1) * kHeadDim);
    }
    if (s0 == kSide * k0) {  // once, with the first reads on their way
      float M = ml[0].x;
#pragma unroll
      for (int i = 1; i < kPer; ++i) M = fmaxf(M, ml[i].x);
      for (int e = 32; e >= 1; e >>= 1) M = fmaxf(M, __shfl_xor(M, e));
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float w = ml[i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[i].x - M);
        weights[wave][lane + 64 * i] = w;
        L += ml[i].y * w;
      }
      for (int e = 32; e >= 1; e >>= 1) L += __shfl_xor(L, e);
      wave_lds_sync();
    }
#pragma unroll
    for (int i = 0; i < IN; ++i) {
      const int s = s0 + kSide * WAVES * i;
      if (s < p.S) {
        if (s + side >= p.S) x[i] = vec{};  // no split: 0 x inf is not 0
        const float w = weights[wave][min(s + side, p.S - 1)];
#pragma unroll
        for (int e = 0; e < W; ++e) o[e] = __builtin_fmaf(x[i][e], w, o[e]);
      }
    }
  }
  if (kSide == 2) {
#pragma unroll
    for (int e = 0; e < W; ++e) o[e] = sum_pair(o[e]);
  }
  if (WAVES > 1) {
    if (side == 0) sums[wave][ln] = o;
    __syncthreads();
    if (k0 != 0) return;
#pragma unroll
    for (int k = 1; k < WAVES; ++k) o += sums[wave + k][ln];
  }
  if (side != 0) return;
  const int kvh = at / p.rows, row = at - kvh * p.rows, tok = row / p.g;
  bvec r;
#pragma unroll
  for (int e = 0; e < W; ++e) r[e] = (__bf16)(o[e] / L);
  *(bvec *)(p.O + (size_t)(kvh * p.g + row - tok * p.g) * p.o_hs + (size_t)tok * p.o_rs + W * ln) = r;
}

// all: rows of all KV heads.  one: splits up to which a wave takes a row, 8 or 12.
inline void launch_join(const AttendOut &p, int64_t all, hipStream_t st, int one = 8) {
  const unsigned fours = (unsigned)((all + kThreads / 64 - 1) / (kThreads / 64));
  if (p.S > 1) {
    if (p.S > 32) join_kernel<4, 16><<<(unsigned)all, kThreads, 0, st>>>(p);
    else if (p.S > one) join_kernel<4, 4><<<(unsigned)all, kThreads, 0, st>>>(p);
    else if (p.S > 8) join_kernel<1, 12><<<fours, kThreads, 0, st>>>(p);
    else join_kernel<1, 8><<<fours, kThreads, 0, st>>>(p);
  }
}

}  // namespace
}  // namespace sa
