// Causal attention of the newest n tokens over the 4-bit cache: O = softmax(scale Q K^T) V, row by row, for n from one token to thousands.  The rows,
// tiles and splits are those of the 8-bit cache (cache_attend.hip); what the 4 bits change is that K goes into the products as it
// is: its codes and scales are the operands of the scaled matrix instructions, and a group of 32 elements is what a lane holds of one.
//   Q, times the softmax scale and log2(e) in fp32, becomes the sum of three codes of 6 bits (e2m3), scales 2^e, 2^(e - 4), 2^(e - 8) for a group of
//   32, the least e with every magnitude <= 7.5 2^e: each takes what the ones before leave, and what the last leaves is 2^-10.9 scales
//   at most, 2^-12.8 of the group's largest.  Codes of 4 and 6 bits multiply at twice the rate of 8 and four times that of 16, so three of them cost
//   three quarters of two codes of 8 bits or of one product in bf16.  (Two codes: chunks 8 % faster, but scores off by 1.4e-3 in the mean.)
//   V has to be multiplied with probabilities, which need bf16: its codes are turned into bf16 on their way into LDS.
// Three kernels, for 16, 32 and 128 query rows a workgroup, and a join of a row's splits; plan_of says which one a call takes.  The first two keep the
// running maximum and sum of an online softmax; with 32 rows the products start at minus a row's reference, so that what comes out is
// the exponent of a probability; with 128 rows probabilities are 2^exponent as it is, and rows that this does not fit are done once more.
#include <algorithm>
#include <cmath>

#include "attend_common.h"
#include "cache4_codes.h"
#include "sa_internal.h"

namespace sa {
namespace {

typedef int i32x6 __attribute__((ext_vector_type(6)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

constexpr int kRowsMany = 128, kRowsFew = 32, kRowsStep = 16;  // query rows of a workgroup
constexpr int kCodes = 3;                                      // of an element of Q

// x / d for 0 <= x < 2^30 as a product: m = ceil(2^(31 + shift) / d) with 2^shift >= d is off by less than d of 2^(31 + shift).  (A division by a number
// that is not known takes some 30 instructions, and what a short call waits for is its code, read once.)
struct Divisor {
  uint32_t m;
  int shift;
};
__device__ inline int divided(int x, Divisor d) { return (int)(__umulhi(2u * (uint32_t)x, d.m) >> d.shift); }
Divisor divisor(int d) {
  int shift = 0;
  while (1 << shift < d) ++shift;
  return {(uint32_t)((((uint64_t)1 << (31 + shift)) + d - 1) / d), shift};
}

struct Attend4Args : AttendOut {
  const uint16_t *Q;
  const uint8_t *K, *V;
  const uint32_t *k_scale, *v_scale;  // a row's four bytes
  int64_t q_hs, q_rs, capacity;
  int tiles;         // row tiles
  Divisor by_g, by_S;
  int turn;          // many rows: row tiles from the last one down, this many, then from the first one up
  int pos, tokens;   // of the first query; in the cache
  float c;           // softmax scale * log2(e), which goes into Q
};

// The codes of 32 elements times c, and their scales, one a byte.
__device__ inline uint32_t cut_query(const uint16_t *at, float c, i32x6 (&code)[kCodes]) {
  uint32_t w[16], top = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) *(uint4 *)&w[4 * k] = ((const uint4 *)at)[k];
  f32x16 even, odd;  // elements 2k, 2k + 1, as the conversion to codes takes them
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    top = max_halves(top, w[k] & 0x7FFF7FFFu);
    even[k] = __uint_as_float(w[k] << 16) * c;
    odd[k] = __uint_as_float(w[k] & 0xFFFF0000u) * c;
  }
  top = max(top & 0xFFFFu, top >> 16);
  // 7.5 = 1.875 * 2^2; the least of the scales is a normal number.  With an infinity or NaN, or one as a product with c, every score is NaN.
  const uint32_t bits = __float_as_uint(fabsf(__uint_as_float(top << 16) * c));
  const int e = max((int)(bits >> 23) - 129 + ((bits & 0x7FFFFFu) > 0x700000u ? 1 : 0), -118);
#pragma unroll
  for (int i = 0; i < kCodes; ++i) {
    const float s = __uint_as_float((uint32_t)(127 + e - 4 * i) << 23);
    const auto q = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, s);
    code[i] = __builtin_bit_cast(i32x6, q);
    if (i + 1 < kCodes) {
      const f32x32 back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(q, s);
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        even[k] -= back[2 * k];
        odd[k] -= back[2 * k + 1];
      }
    }
  }
  const uint32_t b = (uint32_t)(127 + e);
  return bits < 0x7F800000u ? b | (b - 4) << 8 | (b - 8) << 16 : 0x00FFFFFFu;
}

// A workgroup's KV head, split and row tile: KV heads side by side (workgroups go to the XCDs in turn: with 8 KV heads each stays in one L2), then
// splits, then row tiles.  A grid is at most 65535 deep; further row tiles stand beside the KV heads.
struct Place { int kvh, sp, tile; };
__device__ inline Place place_of(const Attend4Args &p) {
  Place at = {(int)blockIdx.x, (int)blockIdx.y, (int)blockIdx.z};
  for (; at.kvh >= p.Hkv; at.kvh -= p.Hkv) at.tile += gridDim.z;
  return at;
}
dim3 grid_of(const Attend4Args &p) {
  const int deep = std::min(p.tiles, 32768);
  return dim3((unsigned)(p.Hkv * ((p.tiles + deep - 1) / deep)), (unsigned)p.S, (unsigned)deep);
}

template <int A_BYTE, int PART>
__device__ inline f32x16 score_product(const uint4 k, const i32x6 (&q)[kCodes], f32x16 acc, uint32_t k_scale, uint32_t q_scale) {
  const i32x8 a = {(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0};
  const i32x8 b = {q[PART][0], q[PART][1], q[PART][2], q[PART][3], q[PART][4], q[PART][5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 2, A_BYTE, (int)k_scale, PART, (int)q_scale);
}

// What a lane has of its row (lane & 31 of the wave's).
struct RowSet {
  i32x6 qc[2][kCodes];
  uint32_t qs[2];
  float m, l;         // the reference of its exponents, the sum of its probabilities
  int row, see, all;  // the row; the last key that it sees; the last that every row of the wave sees
};

template <int N>
struct Int { static constexpr int value = N; };

// Probabilities of pairs N .. N + COUNT - 1 (a pair: accumulators 2N, 2N + 1) as the products take them, in bf16.  PARTS 1: rounded to it, 2^-8 of
// each; 2: a leading part, cut, and the rest, 2^-15, by twice the products.  launch_cache4_attend says which.
template <int N, int COUNT, int HF, int PARTS>
__device__ inline void probabilities(f32x16 (&e)[HF], u32x4 (&pb)[2 * HF][PARTS]) {
#pragma unroll
  for (int n = N; n < N + COUNT; ++n) {
    f32x2 x = {__builtin_amdgcn_exp2f(e[n >> 3][2 * (n & 7)]), __builtin_amdgcn_exp2f(e[n >> 3][2 * (n & 7) + 1])};
    if constexpr (PARTS == 2) {
      const uint32_t a = __float_as_uint(x[0]), b = __float_as_uint(x[1]);
      pb[n >> 2][0][n & 3] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      x[0] -= __uint_as_float(a & 0xFFFF0000u);
      x[1] -= __uint_as_float(b & 0xFFFF0000u);
    }
    pb[n >> 2][PARTS - 1][n & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
  }
}

// Keys that a row does not see, from place lim + 1 (less 4gg) of the tile on.
template <int HF>
__device__ inline void hide(f32x16 (&e)[HF], int lim) {
#pragma unroll
  for (int hf = 0; hf < HF; ++hf)
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (32 * hf + 8 * (k / 4) + k % 4 > lim) e[hf][k] = -INFINITY;
}
// The largest of a row's exponents of a tile.
template <int HF>
__device__ inline float largest(const f32x16 (&e)[HF]) {
  float top[HF];
#pragma unroll
  for (int hf = 0; hf < HF; ++hf) {
    top[hf] = -INFINITY;
#pragma unroll
    for (int k = 0; k < 16; ++k) top[hf] = fmaxf(top[hf], e[hf][k]);
  }
  return max_pair(HF == 1 ? top[0] : fmaxf(top[0], top[HF - 1]));
}

// With 32 and 128 rows a workgroup probabilities are 2^exponent as it is: fp32 and bf16 hold them from 2^-126 to 2^127, so that nothing has to be
// searched, subtracted or rescaled on the way.  V is multiplied by 2^40, so that small values times small probabilities are normal
// numbers: the least of both, 2^-101 and 2^-40, make 2^-101.  (The sum is, too, so that it is as if -40 had been subtracted.)  Where that is not
// enough (a row's sum beyond 2^80 or below 2^-40, or an output that is no number, of V beyond 2^85 or NaN) the rows are done once more, with
// their largest exponents subtracted and V as it is.  With 128 rows a long walk looks at its first tile ahead, and where that is far from 0
// already, subtracts the largest exponents of this tile from the start (2048 tokens of 32 heads at 64K keys, all scores 40 lower: 4000 us without
// the look, 1555 with it; as they come 1510).  Shorter walks, and all with 32 rows, pay for the second pass: scores 40 lower or 60 higher, 200 tokens at 8000 keys
// 40 -> 71 us, 2048 at 8000 220 -> 545; 32 rows, 500 tokens at 500 keys 13.4 -> 23.4, 50 at 5000 16.5 -> 28.
constexpr float kUp = 0x1p40f, kUpRef = -40.f;
__device__ inline bool in_range(float l, const f32x16 (&oacc)[4]) {
  float odd[4] = {};  // 0, or NaN where an output is no number
#pragma unroll
  for (int k = 0; k < 16; ++k)
#pragma unroll
    for (int db = 0; db < 4; ++db) odd[db] = __builtin_fmaf(oacc[db][k], 0.f, odd[db]);
  return l > 0x1p-40f && l < 0x1p80f && odd[0] + odd[1] + odd[2] + odd[3] == 0.f;
}
// A row's sums over `keys` keys hold by themselves, up to the ends of fp32, but they are joined with those of four waves and of up to 256 splits, some of which
// may have been done once more.  So where their mean probability is above 1, its power of two goes into the reference, which is then at most about the largest
// exponent: l is below 2 keys, an output at most that times the largest of V, and a part whose exp2(m - M) is 0, below 2^-126, weighs less than 2^-125 keys.
// l is below 2^121, so that 2^-x is a normal number; 0 (no key), infinite or NaN it stays so.  m + x is rounded where m is no whole
// number, by no more than the scores were.  kLargestOff: the largest exponents of all keys were subtracted, so that there is nothing to move.
constexpr int kLargestOff = 0x7FFFFFFF;
__device__ inline void settle(float &m, float &l, f32x16 (&o)[4], int keys) {
  const int x = max(__builtin_amdgcn_frexp_expf(l) - (32 - __builtin_clz((uint32_t)max(keys, 1))), 0);
  const float s = __builtin_ldexpf(1.f, -x);
  m += (float)x;
  l *= s;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] *= s;
}
// The groups of V that are NaN among the keys first .. first + 63 (rowbad: a byte for each, a bit for each group; 0 from key `end` on), for a row
// that sees keys up to `see`.
__device__ inline void put_nan(const uint8_t *rowbad, int first, int end, int see, f32x16 (&o)[4]) {
  const int lane = threadIdx.x & 63;
  const uint32_t mine = first + lane < end ? rowbad[lane] : 0u;
  for (uint64_t which = __ballot(mine != 0u); which != 0ull; which &= which - 1ull) {
    const int at = __ffsll((unsigned long long)which) - 1;
    const uint32_t bad = (uint32_t)__shfl((int)mine, at);
#pragma unroll
    for (int db = 0; db < 4; ++db)
      if ((bad >> db & 1u) != 0u && first + at <= see)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] = NAN;
  }
}

// Over the four lanes of a row, on each of them.
__device__ inline float over_blocks(float x) {
  x = max_pair(x);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_blocks(float x) {
  x = sum_pair(x);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 32 query rows a workgroup, every wave its own keys, tiles of 32 of them; no barriers on the way.  A lane reads the half row of K that it multiplies
// itself, so that only V goes through LDS, between the products of K.  Bound: one tile after the other, which two waves a SIMD half hide:
// products, their exponentials, V's way through LDS.  500 tokens of 32 heads at 1000 keys 17 us, 50 at 5000 16.5 with the join (8 bits: 19.7 at 500).
template <int PARTS>
__global__ __launch_bounds__(kThreads, 2) void attend4_few_kernel(Attend4Args p) {
  constexpr int KT = 32, WK = kThreads / 64;  // keys per tile, waves
  constexpr int kMasked = 2;                  // tiles that some rows see and others do not, at most: 31 keys
  __shared__ __attribute__((aligned(16))) union {
    uint16_t v[WK][KT * 128];
    float o[WK][32][kHeadDim];
  } lds;
  __shared__ uint8_t rowbad[kMasked * KT];  // keys of the masked tiles: a bit for each group of V that is NaN
  __shared__ float s_m[4][32], s_l[4][32];

  const int tid = threadIdx.x, lane = tid & 63, q = lane & 31, gg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place at_grid = place_of(p);
  if (at_grid.tile >= p.tiles) return;
  const int kvh = at_grid.kvh, sp = at_grid.sp, r0 = (p.tiles - 1 - at_grid.tile) * kRowsFew;  // the longest row tiles first
  const int seen_all = p.pos + divided(r0, p.by_g);     // last key that every row sees
  const int t_masked = (seen_all + 1) / KT;  // first tile that some do not
  const int n_tiles = (p.pos + divided(min(r0 + kRowsFew, p.rows) - 1, p.by_g)) / KT + 1;
  const int per = divided(n_tiles + p.S - 1, p.by_S);
  const int t_begin = min(sp * per, n_tiles), t_end = min(t_begin + per, n_tiles);

  RowSet r;
  r.row = min(r0 + q, p.rows - 1);
  const int tok = divided(r.row, p.by_g), head = kvh * p.g + (r.row - tok * p.g);
  r.see = p.pos + tok;

  const size_t first = (size_t)kvh * p.capacity;
  const uint8_t *__restrict__ Kh = p.K + first * kRow4, *__restrict__ Vh = p.V + first * kRow4;
  const uint32_t *__restrict__ ksh = p.k_scale + first, *__restrict__ vsh = p.v_scale + first;

  uint4 kc[2], vc[2];  // a lane's two groups of K; pieces of V: rows lane / 4 and 16 further, a group each
  uint32_t ks, vs[2];
  unsigned k_row = q, v_row[2] = {(unsigned)lane >> 2, ((unsigned)lane >> 2) + 16};  // of a tile
  auto fetch = [&](int t) {
    if ((t + 1) * KT > p.tokens) {  // the last tile; behind the tokens the last one again: nobody sees it there
      const unsigned last = (unsigned)(p.tokens - 1 - t * KT);
      k_row = min(k_row, last);
      v_row[0] = min(v_row[0], last);
      v_row[1] = min(v_row[1], last);
    }
    const uint8_t *k = Kh + (size_t)t * KT * kRow4, *v = Vh + (size_t)t * KT * kRow4;
    const char *kscale = (const char *)(ksh + (size_t)t * KT), *vscale = (const char *)(vsh + (size_t)t * KT);
    kc[0] = *(const uint4 *)(k + (k_row * kRow4 + 32 * gg));
    kc[1] = *(const uint4 *)(k + (k_row * kRow4 + 32 * gg + 16));
    ks = *(const uint32_t *)(kscale + 4 * k_row);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      vc[i] = *(const uint4 *)(v + (v_row[i] * kRow4 + 16 * (lane & 3)));
      vs[i] = *(const uint32_t *)(vscale + 4 * v_row[i]);
    }
  };
  const int t_first = t_begin + wave;
  if (t_first < t_end) fetch(t_first);

  // Q: the groups 2gg and 2gg + 1 of a row, as the lane's K
  const uint16_t *qrow = p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs + 64 * gg;
#pragma unroll 1
  for (int s = 0; s < 2; ++s) {  // one after the other, in half the code
#pragma unroll
    for (int i = 0; i < kCodes; ++i) r.qc[0][i] = r.qc[1][i];
    r.qs[0] = r.qs[1];
    r.qs[1] = cut_query(qrow + 32 * s, p.c, r.qc[1]);
  }

  unsigned vbase;
  {
    const int x = lane & 15, part = (lane >> 4) & 1, vrow = 4 * gg + (x >> 2);
    vbase = (unsigned)(vrow * 256) | (unsigned)(((2 * part + ((x & 3) >> 1)) ^ ((vrow & 3) * 5)) << 4) | (unsigned)((x & 1) << 3);
  }
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  f32x16 oacc[4];
  f32x4 lacc[2];
  auto run = [&](auto AGAIN) {
    constexpr bool kAgain = decltype(AGAIN)::value != 0;
#pragma unroll
    for (int db = 0; db < 4; ++db) oacc[db] = f32x16{};
    lacc[0] = lacc[1] = f32x4{};
    for (int t = t_first; t < t_end; t += WK) {
      // A row that does not see a key gives it weight 0, and 0 x NaN is not 0: in tiles that only some rows see, groups of V
      // that are NaN stay out of the products and come back at the end for the rows that do see them.
      if (t >= t_masked) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const bool bad = (vs[i] >> (8 * (lane & 3)) & 0xFFu) == kNanScale;
          const uint64_t who = __ballot(bad);
          if ((lane & 3) == 0) rowbad[(t - t_masked) * KT + (lane >> 2) + 16 * i] = (uint8_t)(who >> lane & 15ull);
          if (bad) { vc[i] = make_uint4(0u, 0u, 0u, 0u); vs[i] = 0x7F7F7F7Fu; }
        }
      }
      constexpr float up = kAgain ? 1.f : kUp;
      const float vscale[2] = {scale4(vs[0] >> (8 * (lane & 3)) & 0xFFu) * up, scale4(vs[1] >> (8 * (lane & 3)) & 0xFFu) * up};
      auto put_v = [&](int k) {  // 8 elements of a lane's 64, as bf16 into LDS
        const uint4 &x = vc[k >> 2];
        const uint32_t w = (k & 3) == 0 ? x.x : (k & 3) == 1 ? x.y : (k & 3) == 2 ? x.z : x.w;
        const int at = (lane >> 2) + 16 * (k >> 2);
        *(uint4 *)((char *)lds.v[wave] + at * 256 + (((4 * (lane & 3) + (k & 3)) ^ ((at & 3) * 5)) << 4)) = decode4_8(w, vscale[k >> 2]);
      };
      const uint32_t ksw = ks >> (16 * gg);
      f32x16 e[1];  // S^T = K Q^T (lane = row, accumulator r <-> key 8(r/4) + 4gg + r%4), beside it V on its way into LDS
#define SA_STEP(S, I) \
      e[0] = score_product<S, I>(kc[S], r.qc[S], S == 0 && I == 0 ? f32x16{} : e[0], ksw, r.qs[S]); \
      put_v(4 * S + I); \
      if (I == 0) put_v(4 * S + 3); \
      __builtin_amdgcn_sched_barrier(0);
      SA_STEP(0, 0) SA_STEP(0, 1) SA_STEP(0, 2) SA_STEP(1, 0) SA_STEP(1, 1) SA_STEP(1, 2)
#undef SA_STEP
      if (t + WK < t_end) fetch(t + WK);
      if (kAgain) e[0] -= r.m;
      if ((t + 1) * KT - 1 > seen_all) hide(e, r.see - t * KT - 4 * gg);
      wave_lds_sync();
      u32x4 pb[2][PARTS];
      s16x4 vlo[4], vhi[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        vlo[i] = SA_VTR(lds.v[wave], i & 3, 0);
        vhi[i] = SA_VTR(lds.v[wave], i & 3, 8);
      }
      probabilities<0, 4>(e, pb);
      __builtin_amdgcn_s_setprio(1);
      // The normaliser sums the probabilities as multiplied, so that a row stays a convex combination of its V rows;
      // 4x4x4 products with ones do it on the matrix pipe.
      const s16x4 ones4 = {0x3f80, 0x3f80, 0x3f80, 0x3f80};
      auto step = [&](auto I) {
        constexpr int i = decltype(I)::value, g = i >> 2, db = i & 3;
        const bf16x8 av = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vlo[db], vhi[db], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int x = 0; x < PARTS; ++x) {
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, __builtin_bit_cast(bf16x8, pb[g][x]), oacc[db], 0, 0, 0);
          const s16x8 ps = __builtin_bit_cast(s16x8, pb[g][x]);
          if constexpr (db == 0) lacc[0] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones4, __builtin_shufflevector(ps, ps, 0, 1, 2, 3), lacc[0], 0, 0, 0);
          if constexpr (db == 3) lacc[1] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones4, __builtin_shufflevector(ps, ps, 4, 5, 6, 7), lacc[1], 0, 0, 0);
        }
        if constexpr (i < 4) {
          vlo[db] = SA_VTR(lds.v[wave], db, 16);
          vhi[db] = SA_VTR(lds.v[wave], db, 24);
          probabilities<i + 4, 1>(e, pb);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      step(Int<0>()); step(Int<1>()); step(Int<2>()); step(Int<3>()); step(Int<4>()); step(Int<5>()); step(Int<6>()); step(Int<7>());
      __builtin_amdgcn_s_setprio(0);
      wave_lds_sync();
    }
    r.l = sum_pair(lacc[0][0] + lacc[1][0]);  // the keys of both lanes of a row
  };
  run(Int<0>());
  const bool sees = t_first < t_end && r.see >= t_first * KT;
  const bool again = __any(sees && !in_range(r.l, oacc));
  r.m = sees ? kUpRef : -INFINITY;
  r.l *= kUp;
  if (again) {  // this wave's keys
    float top = -INFINITY;
    auto whole_tiles = [&] {  // after the last tile changed the rows to read
      k_row = q;
      v_row[0] = (unsigned)lane >> 2;
      v_row[1] = ((unsigned)lane >> 2) + 16;
    };
    whole_tiles();
    for (int t = t_first; t < t_end; t += WK) {
      fetch(t);
      const uint32_t ksw = ks >> (16 * gg);
      f32x16 e[1] = {};
#define SA_STEP(S, I) e[0] = score_product<S, I>(kc[S], r.qc[S], e[0], ksw, r.qs[S]);
      SA_STEP(0, 0) SA_STEP(0, 1) SA_STEP(0, 2) SA_STEP(1, 0) SA_STEP(1, 1) SA_STEP(1, 2)
#undef SA_STEP
      hide(e, r.see - t * KT - 4 * gg);
      top = fmaxf(top, largest(e));
    }
    r.m = top == -INFINITY ? 0.f : top;
    whole_tiles();
    fetch(t_first);
    run(Int<1>());
    r.m = top;
  }
  if (t_end > t_masked) {
    __syncthreads();
    for (int t = max(t_begin, t_masked); t < t_end; ++t) {
      if ((t - t_begin) % WK != wave) continue;  // another wave's tile
      put_nan(rowbad + (t - t_masked) * KT, t * KT, (t + 1) * KT, r.see, oacc);
    }
  }
  // Here, not beside the pass above: there the compiler spills the outputs, and a pass that is done once more takes ten times as long.
  settle(r.m, r.l, oacc, again ? kLargestOff : (t_end - t_first + WK - 1) / WK * KT);
  put_waves(p, kvh, r0, sp, r.m, r.l, oacc, &lds.o[0][0][0], s_m, s_l);
}

// Steps: 16 query rows a workgroup, every wave its own keys, tiles of 32 of them.  One v_mfma_scale_f32_16x16x128 takes 16 keys, whole rows of K: a
// lane reads one group of a key and multiplies it with the same group of its query row (lane & 15).  Half the products, exponentials and registers of 32
// rows, so that four waves a SIMD, instead of two, have reads on their way.  Bound: HBM on long caches, one token of 32 heads at 128K keys reads 143 MB in
// 28.0 us (5.1 TB/s), 32.3 to 33.1 with the join (32 rows a workgroup: 39.6); the chain of reads on short ones, 5 tokens of 8 heads on one KV head at 10K keys 9.1.
__global__ __launch_bounds__(kThreads, 4) void attend4_step_kernel(Attend4Args p) {
  constexpr int KT = 32, WK = kThreads / 64, ROWS = kRowsStep;
  constexpr int kMasked = 2;  // tiles that some rows see and others do not, at most: 15 keys
  __shared__ __attribute__((aligned(16))) union {
    uint16_t v[WK][KT * 128];
    float o[WK][ROWS][kHeadDim];
  } lds;
  __shared__ uint8_t rowbad[kMasked * KT];  // keys of the masked tiles: a bit for each group of V that is NaN
  __shared__ float s_m[WK][ROWS], s_l[WK][ROWS];

  const int tid = threadIdx.x, lane = tid & 63, q = lane & 15, b = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place at_grid = place_of(p);
  if (at_grid.tile >= p.tiles) return;
  const int kvh = at_grid.kvh, sp = at_grid.sp, r0 = (p.tiles - 1 - at_grid.tile) * ROWS;  // the longest row tiles first
  const int seen_all = p.pos + divided(r0, p.by_g);     // last key that every row sees
  const int t_masked = (seen_all + 1) / KT;  // first tile that some do not
  const int n_tiles = (p.pos + divided(min(r0 + ROWS, p.rows) - 1, p.by_g)) / KT + 1;
  const int per = divided(n_tiles + p.S - 1, p.by_S);
  const int t_begin = min(sp * per, n_tiles), t_end = min(t_begin + per, n_tiles);

  // this lane's row, and the last key that it sees
  const int row = min(r0 + q, p.rows - 1), tok = divided(row, p.by_g), head = kvh * p.g + (row - tok * p.g), see = p.pos + tok;

  const size_t first = (size_t)kvh * p.capacity;
  const uint8_t *__restrict__ Kh = p.K + first * kRow4, *__restrict__ Vh = p.V + first * kRow4;
  const uint32_t *__restrict__ ksh = p.k_scale + first, *__restrict__ vsh = p.v_scale + first;

  uint4 kc[2], vc[2];  // a group of the keys q and q + 16; pieces of V: rows lane / 4 and 16 further, a group each
  uint32_t ks[2], vs[2];
  unsigned k_row[2] = {(unsigned)q, (unsigned)q + 16}, v_row[2] = {(unsigned)lane >> 2, ((unsigned)lane >> 2) + 16};  // of a tile
  auto fetch = [&](int t) {
    if ((t + 1) * KT > p.tokens) {  // the last tile; behind the tokens the last one again: nobody sees it there
      const unsigned last = (unsigned)(p.tokens - 1 - t * KT);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        k_row[i] = min(k_row[i], last);
        v_row[i] = min(v_row[i], last);
      }
    }
    const uint8_t *k = Kh + (size_t)t * KT * kRow4, *v = Vh + (size_t)t * KT * kRow4;
    const char *kscale = (const char *)(ksh + (size_t)t * KT), *vscale = (const char *)(vsh + (size_t)t * KT);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      kc[i] = *(const uint4 *)(k + (k_row[i] * kRow4 + 16 * b));
      vc[i] = *(const uint4 *)(v + (v_row[i] * kRow4 + 16 * (lane & 3)));
      ks[i] = *(const uint32_t *)(kscale + 4 * k_row[i]);
      vs[i] = *(const uint32_t *)(vscale + 4 * v_row[i]);
    }
  };
  int t = t_begin + wave;
  if (t < t_end) fetch(t);

  i32x6 qc[kCodes];
  const uint32_t qs = cut_query(p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs + 32 * b, p.c, qc);

  f32x4 oacc[8] = {};  // lane = row, accumulator r of piece db <-> element 16db + 4b + r
  float m_run = -INFINITY, l_run = 0.f;
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  // V of a tile in LDS: key r in 256 bytes, the 16-byte chunk c at c ^ place(r), so that the stores of 16 lanes (four keys, a group of each) and the
  // transposing reads of 64 (16 keys, 16 elements of each) spread over all banks.
  auto place = [](int r) { return (r & 3) * 5 ^ (r >> 2 & 1) << 1; };
  unsigned vbase;
  {
    const int r = lane & 15, vrow = 4 * b + (r >> 2);
    vbase = (unsigned)(vrow * 256) | (unsigned)(((r & 3) >> 1 ^ place(vrow)) << 4) | (unsigned)((r & 1) << 3);
  }
  for (; t < t_end; t += WK) {
    // A row that does not see a key gives it weight 0, and 0 x NaN is not 0: in tiles that only some rows see, groups of V
    // that are NaN stay out of the products and come back at the end for the rows that do see them.
    if (t >= t_masked) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const bool bad = (vs[i] >> (8 * (lane & 3)) & 0xFFu) == kNanScale;
        const uint64_t who = __ballot(bad);
        if ((lane & 3) == 0) rowbad[(t - t_masked) * KT + (lane >> 2) + 16 * i] = (uint8_t)(who >> lane & 15ull);
        if (bad) { vc[i] = make_uint4(0u, 0u, 0u, 0u); vs[i] = 0x7F7F7F7Fu; }
      }
    }
    f32x4 e[2];  // exponents: lane = row, accumulator r of half i <-> key 16i + 4b + r
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const i32x8 a = {(int)kc[i].x, (int)kc[i].y, (int)kc[i].z, (int)kc[i].w, 0, 0, 0, 0};
      const int scale = (int)(ks[i] >> (8 * b));
      const f32x4 zero = {};
      auto codes = [&](int k) { return i32x8{qc[k][0], qc[k][1], qc[k][2], qc[k][3], qc[k][4], qc[k][5], 0, 0}; };
      e[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, codes(0), zero, 4, 2, 0, scale, 0, (int)qs);
      e[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, codes(1), e[i], 4, 2, 0, scale, 1, (int)qs);
      e[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, codes(2), e[i], 4, 2, 0, scale, 2, (int)qs);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float s = scale4(vs[i] >> (8 * (lane & 3)) & 0xFFu);
      const uint32_t w[4] = {vc[i].x, vc[i].y, vc[i].z, vc[i].w};
      const int r = (lane >> 2) + 16 * i;
#pragma unroll
      for (int k = 0; k < 4; ++k) *(uint4 *)((char *)lds.v[wave] + r * 256 + (((4 * (lane & 3) + k) ^ place(r)) << 4)) = decode4_8(w[k], s);
    }
    const int now = t;
    if (t + WK < t_end) fetch(t + WK);
    wave_lds_sync();
    if ((now + 1) * KT - 1 > seen_all) {
      const int lim = see - now * KT - 4 * b;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * i + r > lim) e[i][r] = -INFINITY;
    }
    float top = fmaxf(fmaxf(fmaxf(e[0][0], e[0][1]), fmaxf(e[0][2], e[0][3])), fmaxf(fmaxf(e[1][0], e[1][1]), fmaxf(e[1][2], e[1][3])));
    // The reference moves only when some row's exponents grew beyond it by more than 8, see absorb_exponents
    if (__any(top - m_run > 8.f)) {
      top = fmaxf(m_run, over_blocks(top));
      const float alpha = __builtin_amdgcn_exp2f(m_run - (top == -INFINITY ? 0.f : top));
      m_run = top;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < 8; ++db) oacc[db] *= alpha;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    u32x4 lead, rest;  // the probabilities in two parts: cut, and what that leaves
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const float x = __builtin_amdgcn_exp2f(e[i][r] - ref), y = __builtin_amdgcn_exp2f(e[i][r + 1] - ref);
        l_run += x;
        l_run += y;
        const uint32_t wx = __float_as_uint(x), wy = __float_as_uint(y);
        const f32x2 left = {x - __uint_as_float(wx & 0xFFFF0000u), y - __uint_as_float(wy & 0xFFFF0000u)};
        lead[2 * i + r / 2] = __builtin_amdgcn_perm(wy, wx, 0x07060302u);
        rest[2 * i + r / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(left, bf16x2));
      }
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const unsigned at = vbase ^ (unsigned)(db << 5);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((const char *)lds.v[wave] + at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((const char *)lds.v[wave] + at + 16 * 256));
      const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      oacc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, lead), oacc[db], 0, 0, 0);
      oacc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, rest), oacc[db], 0, 0, 0);
    }
    wave_lds_sync();
  }
  if (t_end > t_masked) {
    __syncthreads();
    for (int t = max(t_begin, t_masked); t < t_end; ++t) {
      if ((t - t_begin) % WK != wave) continue;  // another wave's tile
      const uint32_t mine = lane < KT ? rowbad[(t - t_masked) * KT + lane] : 0u;
      for (uint64_t which = __ballot(mine != 0u); which != 0ull; which &= which - 1ull) {
        const int at = __ffsll((unsigned long long)which) - 1;
        const uint32_t bad = (uint32_t)__shfl((int)mine, at);
#pragma unroll
        for (int db = 0; db < 8; ++db)
          if ((bad >> (db / 2) & 1u) != 0u && t * KT + at <= see) oacc[db] = f32x4{NAN, NAN, NAN, NAN};
      }
    }
  }
  const float l_row = sum_blocks(l_run);  // the keys of the four lanes of a row

  // ---- the four waves' sums of the same rows, through the LDS of the tiles: O / l in bf16, or the split's sums
  __syncthreads();
  if (b == 0) { s_m[wave][q] = m_run; s_l[wave][q] = l_row; }
#pragma unroll
  for (int db = 0; db < 8; ++db)
    *(f32x4 *)&lds.o[wave][q][(16 * db + 4 * b) ^ (q & 7) << 2] = oacc[db];
  __syncthreads();
  const int mr = tid >> 4, d0 = (tid & 15) * 8;  // 8 outputs of a row each
  const int orow = r0 + mr;
  if (orow >= p.rows) return;
  float M = -INFINITY, L = 0.f, w[WK];
#pragma unroll
  for (int k = 0; k < WK; ++k) M = fmaxf(M, s_m[k][mr]);
#pragma unroll
  for (int k = 0; k < WK; ++k) {
    w[k] = s_m[k][mr] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[k][mr] - M);
    L += s_l[k][mr] * w[k];
  }
  const size_t slot = ((size_t)kvh * p.rows + orow) * p.S + sp;
  const int otok = divided(orow, p.by_g);
  uint16_t *o = p.O + (size_t)(kvh * p.g + orow - otok * p.g) * p.o_hs + (size_t)otok * p.o_rs;
  if (p.S > 1 && d0 == 0) p.ml[slot] = make_float2(M, L);
  const float inv = p.S > 1 ? 1.f : 1.f / L;
  f32x4 x[2] = {};
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int k = 0; k < WK; ++k) x[i] += *(const f32x4 *)&lds.o[k][mr][(d0 + 4 * i) ^ (mr & 7) << 2] * w[k];
  if (p.S > 1) {
#pragma unroll
    for (int i = 0; i < 2; ++i) *(f32x4 *)(p.part + slot * kHeadDim + d0 + 4 * i) = x[i];
  } else {
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 u = {(__bf16)(x[i / 2][2 * (i & 1)] * inv), (__bf16)(x[i / 2][2 * (i & 1) + 1] * inv)};
      y[i] = __builtin_bit_cast(uint32_t, u);
    }
    *(uint4 *)(o + d0) = make_uint4(y[0], y[1], y[2], y[3]);
  }
}

// K Q^T of half a tile (the codes of d-slab S) for both halves of the keys, product I of kCodes.
template <int S, int I>
__device__ inline void score_pair(const uint4 (&kf)[2][2], const RowSet &r, f32x16 (&e)[2], const uint32_t (&ks)[2]) {
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) e[hf] = score_product<S, I>(kf[S][hf], r.qc[S], S == 0 && I == 0 ? f32x16{} : e[hf], ks[hf], r.qs[S]);
}

// K Q^T of a tile.
__device__ inline void scores(const uint4 (&kf)[2][2], const RowSet &r, f32x16 (&e)[2], const uint32_t (&ks)[2]) {
  score_pair<0, 0>(kf, r, e, ks);
  score_pair<0, 1>(kf, r, e, ks);
  score_pair<0, 2>(kf, r, e, ks);
  score_pair<1, 0>(kf, r, e, ks);
  score_pair<1, 1>(kf, r, e, ks);
  score_pair<1, 2>(kf, r, e, ks);
}

// Many rows: four waves of 32 query rows each, which share tiles of 64 keys.  K goes from memory into LDS as it is (the LDS DMA, no registers), V
// in bf16, from registers that were read a tile ahead; beside the products of a tile, V of the next one.  Bound: the matrix pipe at the power
// limit, 2048 tokens of 32 heads at 64K keys 1505 to 1560 us by card, 1.44 to 1.39 PFLOP/s (8 bits: 1650 to 1790; a library product of bf16 1.35), with
// the clock at 2.0 GHz.  64 rows a wave, eight waves that share V or the keys of a tile, and a tile's products begun beside the last one's end were slower.
__global__ __launch_bounds__(kThreads, 2) void attend4_rows_kernel(Attend4Args p) {
  constexpr int KT = 64, ROWS = kRowsMany;
  constexpr int kLong = 256;  // tiles of a walk that is worth a look ahead
  constexpr int kMasked = 3;  // tiles that some rows see and others do not, at most: 127 keys
  __shared__ __attribute__((aligned(16))) uint8_t Ks[2][KT * kRow4];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[2][KT * 128];
  __shared__ uint8_t rowbad[kMasked * KT];  // keys of the masked tiles: a bit for each group of V that is NaN

  const int tid = threadIdx.x, lane = tid & 63, q = lane & 31, gg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place at_grid = place_of(p);
  if (at_grid.tile >= p.tiles) return;
  const int kvh = at_grid.kvh, sp = at_grid.sp, rt = at_grid.tile < p.turn ? p.tiles - 1 - at_grid.tile : at_grid.tile - p.turn;
  const int r0 = rt * ROWS, r_last = min(r0 + ROWS, p.rows) - 1;
  const int seen_all = p.pos + divided(r0, p.by_g);                // last key that every row of the workgroup sees
  const int t_masked = (seen_all + 1) / KT;             // first tile that some do not
  const int n_tiles = (p.pos + divided(r_last, p.by_g)) / KT + 1;  // tiles that some row sees
  const int per = divided(n_tiles + p.S - 1, p.by_S);
  const int t_begin = min(sp * per, n_tiles), t_end = min(t_begin + per, n_tiles);

  const size_t first = (size_t)kvh * p.capacity;
  const uint8_t *__restrict__ Kh = p.K + first * kRow4, *__restrict__ Vh = p.V + first * kRow4;
  const uint32_t *__restrict__ ksh = p.k_scale + first, *__restrict__ vsh = p.v_scale + first;

  // ---- what a thread reads of a tile, from the tile's first byte on; behind the tokens the last row again: nobody sees it there.
  // K: 64 rows of 64 bytes, the 16-byte chunk c of row r in place c ^ (r / 4) % 4, so that b128 reads of 16 rows hit 64 banks (the
  // lane that owns place x of row r reads chunk x ^ (r / 4) % 4).  V: a group of 32 codes of row vrow.  Scales of K: of the keys q and q + 32.
  const unsigned ldsK = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)&Ks[0][0] + wave * 1024;
  const int vrow = tid >> 2, vg = tid & 3;
  unsigned k_at, v_at, vs_at, ks_at[2];
  auto offsets = [&](int rows) {
    k_at = (unsigned)(min(16 * wave + (lane >> 2), rows - 1) * kRow4 + (((lane & 3) ^ (lane >> 4)) << 4));
    const int r = min(vrow, rows - 1);
    v_at = (unsigned)(r * kRow4 + vg * 16);
    vs_at = 4u * (unsigned)r;
    ks_at[0] = 4u * (unsigned)min(q, rows - 1);
    ks_at[1] = 4u * (unsigned)min(q + 32, rows - 1);
  };
  const int n_whole = p.tokens / KT;  // tiles without a row behind the tokens
  auto issue_k = [&](int t, int buf) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(k_at), "s"(Kh + (size_t)t * KT * kRow4),
                 "s"(ldsK + (unsigned)(buf * KT * kRow4)) : "memory");
  };
  uint32_t kn[2], ks[2];  // as read, and as the products take them
  auto fetch_ks = [&](int t) {
    const char *at = (const char *)(ksh + (size_t)t * KT);
    kn[0] = *(const uint32_t *)(at + ks_at[0]);
    kn[1] = *(const uint32_t *)(at + ks_at[1]);
  };
  const unsigned kbase = (unsigned)(q * kRow4) | (unsigned)(((2 * gg) ^ (q >> 2 & 3)) << 4);
  uint4 kf[2][2];  // [d-slab][half of the keys]
  auto read_k = [&](int buf) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) kf[s][hf] = *(const uint4 *)((const char *)&Ks[0][0] + (buf * KT + 32 * hf) * kRow4 + (kbase ^ (unsigned)(s << 4)));
  };
  uint4 vc;
  uint32_t vs;
  auto fetch_v = [&](int t) {
    vc = *(const uint4 *)(Vh + (size_t)t * KT * kRow4 + v_at);
    vs = *(const uint32_t *)((const char *)(vsh + (size_t)t * KT) + vs_at);
  };
  char *const vput = (char *)&Vs[0][0] + vrow * 256;
  const unsigned vswz = (unsigned)(4 * vg ^ (vrow & 3) * 5) << 4;
  auto put_v = [&](int buf, int k, float scale) {
    const uint32_t w = k == 0 ? vc.x : k == 1 ? vc.y : k == 2 ? vc.z : vc.w;
    *(uint4 *)(vput + buf * KT * 256 + (vswz ^ (unsigned)(k << 4))) = decode4_8(w, scale);
  };
  // A row that does not see a key gives it weight 0, and 0 x NaN is not 0: in tiles that only some rows see, groups of V
  // that are NaN stay out of the products and come back at the end for the rows that do see them.
  auto screen = [&](int t) {
    const bool bad = (vs >> (8 * vg) & 0xFFu) == kNanScale;
    const uint64_t who = __ballot(bad);
    if (vg == 0) rowbad[(t - t_masked) * KT + vrow] = (uint8_t)(who >> lane & 15ull);
    if (bad) { vc = make_uint4(0u, 0u, 0u, 0u); vs = 0x7F7F7F7Fu; }
  };
  unsigned vbase;
  {
    const int r = lane & 15, part = (lane >> 4) & 1, vr = 4 * gg + (r >> 2);
    vbase = (unsigned)(vr * 256) | (unsigned)(((2 * part + ((r & 3) >> 1)) ^ ((vr & 3) * 5)) << 4) | (unsigned)((r & 1) << 3);
  }
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

  auto begin = [&] {
    offsets(t_begin < n_whole ? KT : p.tokens - t_begin * KT);
    issue_k(t_begin, 0);
    fetch_v(t_begin);
    fetch_ks(t_begin);
  };
  if (t_begin < t_end) begin();
  RowSet r;
  int head, tok;
  {
    const int lo = min(r0 + 32 * wave, p.rows - 1);
    r.row = min(lo + q, p.rows - 1);
    tok = divided(r.row, p.by_g);
    head = kvh * p.g + (r.row - tok * p.g);
    r.see = p.pos + tok;
    r.all = p.pos + divided(lo, p.by_g);
    const uint16_t *qrow = p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs + 64 * gg;
#pragma unroll 1
    for (int s = 0; s < 2; ++s) {  // one after the other, in half the code
#pragma unroll
      for (int i = 0; i < kCodes; ++i) r.qc[0][i] = r.qc[1][i];
      r.qs[0] = r.qs[1];
      r.qs[1] = cut_query(qrow + 32 * s, p.c, r.qc[1]);
    }
  }
  const bool idle = r0 + 32 * wave >= p.rows;  // a wave without rows only turns its part of V into bf16
  f32x16 oacc[4];
  f32x4 lacc[2];
  auto run = [&](auto AGAIN) {
    constexpr bool kAgain = decltype(AGAIN)::value != 0;
    constexpr float up = kAgain ? 1.f : kUp;
#pragma unroll
    for (int db = 0; db < 4; ++db) oacc[db] = f32x16{};
    lacc[0] = lacc[1] = f32x4{};
    if (t_begin < t_end) {
      if (t_begin >= t_masked) screen(t_begin);
      {
        const float s = scale4(vs >> (8 * vg) & 0xFFu) * up;
#pragma unroll
        for (int k = 0; k < 4; ++k) put_v(0, k, s);
      }
      // What a tile begins with, for every wave: K of it has landed, and V of the next one; after the barrier both buffers of the tile hold it
      // and every wave is done with the tile before.  The scale of V of the next tile.
      auto turn = [&](int t, int cur) {
        __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
        __syncthreads();
        read_k(cur);
        ks[0] = kn[0] >> (16 * gg);
        ks[1] = kn[1] >> (16 * gg);
        if (t + 1 < t_end) {
          issue_k(t + 1, cur ^ 1);
          fetch_ks(t + 1);
          if (t + 1 >= t_masked) screen(t + 1);
        }
        return scale4(vs >> (8 * vg) & 0xFFu) * up;
      };
      auto fetch_next = [&](int t) {
        if (t >= t_end) return;
        if (t >= n_whole) offsets(p.tokens - t * KT);  // K and its scales follow
        fetch_v(t);
      };
      fetch_next(t_begin + 1);
      auto tile = [&](auto CUR, int t) {
        constexpr int cur = decltype(CUR)::value;
        const int j0 = t * KT;
        const float scale = turn(t, cur);
        // S^T = K Q^T; beside it V of the next tile becomes bf16 (behind the last tile what is left in the registers: nobody reads it)
        f32x16 e[2];
        __builtin_amdgcn_sched_barrier(0);
#define SA_STEP(S, I, K) \
        score_pair<S, I>(kf, r, e, ks); \
        if constexpr ((K) < 4) put_v(cur ^ 1, K, scale); \
        asm volatile("" : "+v"(e[0]), "+v"(e[1])); \
        __builtin_amdgcn_sched_barrier(0);
        SA_STEP(0, 0, 0) SA_STEP(0, 1, 1) SA_STEP(0, 2, 2) SA_STEP(1, 0, 3) SA_STEP(1, 1, 4) SA_STEP(1, 2, 4)
#undef SA_STEP
        fetch_next(t + 2);
        if (kAgain) {
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            e[0][k] -= r.m;
            e[1][k] -= r.m;
          }
        }
        if (j0 + KT - 1 > r.all) hide(e, r.see - j0 - 4 * gg);
        u32x4 pb[4][1];
        s16x4 vlo[4], vhi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vlo[i] = SA_VTR(Vs[cur], i & 3, 0);
          vhi[i] = SA_VTR(Vs[cur], i & 3, 8);
        }
        probabilities<0, 4>(e, pb);
        __builtin_amdgcn_s_setprio(1);
        // The normaliser sums the probabilities as multiplied, so that a row stays a convex combination of its V rows;
        // 4x4x4 products with ones do it on the matrix pipe.
        const s16x4 ones4 = {0x3f80, 0x3f80, 0x3f80, 0x3f80};
        auto step = [&](auto I) {
          constexpr int i = decltype(I)::value, g = i >> 2, db = i & 3;
          const bf16x8 av = __builtin_bit_cast(bf16x8, __builtin_shufflevector(vlo[db], vhi[db], 0, 1, 2, 3, 4, 5, 6, 7));
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, __builtin_bit_cast(bf16x8, pb[g][0]), oacc[db], 0, 0, 0);
          const s16x8 ps = __builtin_bit_cast(s16x8, pb[g][0]);
          if constexpr (db == 0) lacc[0] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones4, __builtin_shufflevector(ps, ps, 0, 1, 2, 3), lacc[0], 0, 0, 0);
          if constexpr (db == 3) lacc[1] = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(ones4, __builtin_shufflevector(ps, ps, 4, 5, 6, 7), lacc[1], 0, 0, 0);
          if constexpr (i + 4 < 16) {
            vlo[db] = SA_VTR(Vs[cur], db, 16 * ((i + 4) >> 2));
            vhi[db] = SA_VTR(Vs[cur], db, 16 * ((i + 4) >> 2) + 8);
          }
          if constexpr (i < 12) probabilities<i + 4, 1>(e, pb);
          __builtin_amdgcn_sched_barrier(0);
        };
        step(Int<0>()); step(Int<1>()); step(Int<2>()); step(Int<3>()); step(Int<4>()); step(Int<5>()); step(Int<6>()); step(Int<7>());
        step(Int<8>()); step(Int<9>()); step(Int<10>()); step(Int<11>()); step(Int<12>()); step(Int<13>()); step(Int<14>()); step(Int<15>());
        __builtin_amdgcn_s_setprio(0);
      };
      if (idle) {
        for (int t = t_begin; t < t_end; ++t) {
          const int cur = (t - t_begin) & 1;
          const float scale = turn(t, cur);
#pragma unroll
          for (int k = 0; k < 4; ++k) put_v(cur ^ 1, k, scale);
          fetch_next(t + 2);
        }
      } else {
        for (int t = t_begin; t < t_end; t += 2) {
          tile(Int<0>(), t);
          if (t + 1 < t_end) tile(Int<1>(), t + 1);
        }
      }
    }
    r.l = sum_pair(lacc[0][0] + lacc[1][0]);  // the keys of both lanes of a row
  };
  auto some_wave = [](bool x) { return __builtin_amdgcn_readfirstlane(__syncthreads_or(x)) != 0; };
  auto refer = [&](int t_top) {  // to the largest exponents of the tiles up to t_top; the walk begins anew
    float top = -INFINITY;
    offsets(t_begin < n_whole ? KT : p.tokens - t_begin * KT);
    for (int t = t_begin; t < t_top; ++t) {
      if (t >= n_whole) offsets(p.tokens - t * KT);
      __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): what was issued before goes to the same place
      __syncthreads();
      issue_k(t, 0);
      fetch_ks(t);
      __builtin_amdgcn_s_waitcnt(0x0F70);
      __syncthreads();
      ks[0] = kn[0] >> (16 * gg);
      ks[1] = kn[1] >> (16 * gg);
      read_k(0);
      f32x16 e[2];
      scores(kf, r, e, ks);
      hide(e, r.see - t * KT - 4 * gg);
      top = fmaxf(top, largest(e));
    }
    __syncthreads();
    begin();
    r.m = top;
  };
  const bool sees = !idle && t_begin < t_end && r.see >= t_begin * KT;
  bool low = false;  // whether a long walk begins with exponents that do not fit
  if (t_end - t_begin >= kLong) {
    refer(t_begin + 1);
    low = some_wave(sees && r.m > -INFINITY && (r.m < -20.f || r.m > 40.f));
  }
  bool again = low;
  if (!low) {
    run(Int<0>());
    again = some_wave(sees && !in_range(r.l, oacc));
    r.m = sees ? kUpRef : -INFINITY;
    r.l *= kUp;
  }
  int keys = (t_end - t_begin) * KT;
  for (int t_top = low ? t_begin + 1 : t_end; again; t_top = t_end) {
    if (t_top == t_end) keys = kLargestOff;
    refer(t_top);
    if (r.m == -INFINITY) r.m = 0.f;
    run(Int<1>());
    if (r.l == 0.f) r.m = -INFINITY;
    again = t_top < t_end && some_wave(sees && !in_range(r.l, oacc));
  }
  if (t_end > t_masked) {
    __syncthreads();
    for (int t = max(t_begin, t_masked); t < t_end; ++t) put_nan(rowbad + (t - t_masked) * KT, t * KT, (t + 1) * KT, r.see, oacc);
  }
  settle(r.m, r.l, oacc, keys);
  if (r0 + 32 * wave + q < p.rows) put_row(p, kvh, r.row, head, tok, sp, gg, r.m, r.l, oacc);
}

// Rows x splits that the scratch holds: two workgroups of 128 rows a compute unit, as for the 8-bit cache.
size_t max_slots(const Shape &sh) { return (size_t)sh.n_cu * 256; }

// Which kernel, and into how many splits the keys go: the least of an estimate over the three kernels and over splits that fill a quarter of the card, a
// half, .. all that a compute unit holds at once.  The terms were fitted (us) to some 13000 measurements of 1500 drawn shapes of 4 to 64
// heads, 1 to 2048 tokens and up to 131072 keys, in recorded loops; over these, the 1100 that the terms were fitted to among them, the choice is 0.5 % slower than the
// best of all kernels and splits in the mean, and 21.5 % at worst.  There is no term for the rate of memory or the power limit, so that for the longest calls it is less than the time.
//                                              16 rows   32 rows, up to 64 in all   32 rows   128 rows
//   start and end                              3.45      5.65                       5.65      5.2
//   keys of a round of a workgroup's waves     128       128                        128       64
//   a round, up to a workgroup a compute unit  0.92      1.0                        0.73      0.95
//   more of that for each further one          0.28      0.75                       0.8       0.3
//   more at the start for each further one     1.25      0.37                       0.37
//   workgroups a compute unit at once          4         2                          2         2
//   further ones: as many as on average; with 16 and 128 rows halfway from there to the compute units that have the most
//   more than that: their number times this, of which rows see less than the longest one, and 0.6 of a start
//   a join: its launch 2.7, and 1 KB written and read for each row and split
struct Plan { int rows, S; };
Plan plan_of(const Shape &sh, int rows, int tokens, int pos) {
  struct Kernel { int rows, keys, waves, most; float start, more_start, round, more_round, full; };  // keys of a tile, waves that share out the tiles
  const bool parts = rows <= 2 * kRowsFew;
  const Kernel kernels[3] = {{kRowsStep, 32, 4, 4, 3.45f, 1.25f, 0.92f, 0.28f, 0.5f},
                             {kRowsFew, 32, 4, 2, 5.65f, 0.37f, parts ? 1.f : 0.73f, parts ? 0.75f : 0.8f, 0.f},
                             {kRowsMany, 64, 1, 2, 5.2f, 0.f, 0.95f, 0.3f, 0.5f}};
  const float mean = 0.5f + 0.5f * pos / tokens;  // keys that a row sees, against all
  const int64_t all = (int64_t)rows * sh.Hkv;
  Plan best = {kRowsStep, 1};
  float least = INFINITY;
  for (const Kernel &k : kernels) {
    const int64_t wgs = (rows + k.rows - 1) / k.rows * (int64_t)sh.Hkv;
    const int tiles = (tokens + k.keys - 1) / k.keys;
    const int top = (int)std::min<int64_t>(std::min(tiles / k.waves + 1, kMaxSplits), std::max<int64_t>(1, (int64_t)max_slots(sh) / all));
    for (int quarters : {0, 1, 2, 3, 4, 6, 8, 12, 16}) {  // of a workgroup a compute unit; 0: no splits
      const int64_t fill = quarters * (int64_t)sh.n_cu / (4 * wgs);
      if (quarters > 4 * k.most || (quarters > 0 && fill <= 1)) continue;
      const int S0 = (int)std::max<int64_t>(1, std::min<int64_t>(fill, top));
      const int share = (tiles + S0 - 1) / S0, S = (tiles + share - 1) / share, per = (share + k.waves - 1) / k.waves;
      const float load = (float)wgs * S / sh.n_cu;
      const float beside = std::min(std::max(load + k.full * (std::ceil(load) - load) - 1.f, 0.f), k.most - 1.f);
      const float body = k.more_start * beside + per * (k.round + k.more_round * beside);
      float t = k.start + body;
      if (load > k.most) t = std::max(t, load / k.most * (0.6f * k.start + k.more_start * beside + per * (k.round + k.more_round * beside) * mean));
      if (S > 1) t += 2.7f + all * S * 0.0003f;
      if (t < least) { least = t; best = {k.rows, S}; }
    }
  }
  return best;
}

}  // namespace

void cache4_attend_plan(const Shape &sh, int n, int pos, int *rows, int *splits) {
  const Plan plan = plan_of(sh, sh.g * n, pos + n, pos);
  *rows = plan.rows;
  *splits = plan.S;
}

hipError_t launch_cache4_attend(const Shape &sh, const sa_cache4 &c, sa_rows Q, int n, int pos, sa_rows O, void *scratch, hipStream_t st) {
  Attend4Args a;
  a.Q = (const uint16_t *)Q.data; a.O = (uint16_t *)O.data;
  a.K = (const uint8_t *)c.k; a.V = (const uint8_t *)c.v;
  a.k_scale = (const uint32_t *)c.k_scale; a.v_scale = (const uint32_t *)c.v_scale;
  a.q_hs = Q.head_stride; a.q_rs = Q.row_stride; a.o_hs = O.head_stride; a.o_rs = O.row_stride;
  a.capacity = c.capacity;
  a.g = sh.g; a.Hkv = sh.Hkv; a.rows = sh.g * n;
  a.pos = pos; a.tokens = pos + n;
  a.c = sh.scale * 1.4426950408889634f;
  const Plan plan = plan_of(sh, a.rows, a.tokens, pos);
  a.S = plan.S;
  a.tiles = (a.rows + plan.rows - 1) / plan.rows;
  const int64_t wgs = (int64_t)a.tiles * sh.Hkv;
  a.turn = a.tiles;
  if (plan.rows == kRowsMany && wgs * a.S > sh.n_cu && wgs * a.S <= 2 * sh.n_cu) a.turn = std::max(1, (int)(sh.n_cu / (sh.Hkv * a.S)));
  const int64_t all = (int64_t)a.rows * sh.Hkv;
  a.ml = (float2 *)scratch;
  a.part = (float *)((char *)scratch + max_slots(sh) * 8);
  a.by_g = divisor(a.g);
  a.by_S = divisor(a.S);
  const dim3 grid = grid_of(a);
  if (plan.rows == kRowsStep) attend4_step_kernel<<<grid, kThreads, 0, st>>>(a);
  else if (plan.rows == kRowsFew && a.rows <= 2 * kRowsFew) attend4_few_kernel<2><<<grid, kThreads, 0, st>>>(a);
  else if (plan.rows == kRowsFew) attend4_few_kernel<1><<<grid, kThreads, 0, st>>>(a);
  else attend4_rows_kernel<<<grid, kThreads, 0, st>>>(a);
  // Many rows of 9 to 12 splits: a wave a row, against four of them (us, whole calls, 33 shapes): up to 400 rows 0 to 0.3 slower (64 rows, 12 splits 7.6 instead of 7.3), at 768
  // the same (14.7, 14.8), from 2500 on 0.5 to 1.6 faster (5120 rows, 12 splits 42.6 instead of 43.2; 6400, 9 splits 49.2 instead of 50.9).
  launch_join(a, all, st, all >= 1024 ? 12 : 8);
  return hipGetLastError();
}

}  // namespace sa
