// Causal attention of the newest n tokens over the 4-bit cache: O = softmax(scale Q K^T) V, row by row, with the running maximum and sum of an
// online softmax, for n from one token to thousands.  The rows, tiles and splits are those of the 8-bit cache (cache_attend.hip); what the 4 bits
// change is that K goes into the products as it is: its codes and scales are the operands of the scaled matrix instructions, and
// a group of 32 elements is what a lane holds of one.
//   Q, in bf16, becomes the sum of three codes of 6 bits (e2m3), scales 2^e, 2^(e - 4), 2^(e - 8) for a group of 32, the least e with
//   every |q| <= 7.5 2^e: each takes what the ones before leave, all steps exact but the last, which leaves out 2^-12 scales at most, 2^-13.9
//   of the group's largest.  Codes of 4 and 6 bits multiply at twice the rate of 8 and four times that of 16, so three of them cost
//   three quarters of two codes of 8 bits or of one product in bf16.
//   V has to be multiplied with probabilities, which need bf16: its codes are turned into bf16 on their way into LDS.
#include <algorithm>
#include <cmath>

#include "attend_common.h"
#include "cache4_codes.h"
#include "sa_internal.h"

namespace sa {
namespace {

typedef int i32x6 __attribute__((ext_vector_type(6)));
typedef __bf16 bf16x32 __attribute__((ext_vector_type(32)));
typedef float f32x32 __attribute__((ext_vector_type(32)));

constexpr int kRowsMany = 128, kRowsFew = 32;  // query rows of a workgroup

struct Attend4Args : AttendOut {
  const uint16_t *Q;
  const uint8_t *K, *V;
  const uint32_t *k_scale, *v_scale;  // a row's four bytes
  int64_t q_hs, q_rs, capacity;
  int tiles;         // row tiles
  int turn;          // many rows: row tiles from the last one down, this many, then from the first one up
  int pos, tokens;   // of the first query; in the cache
  float c;           // softmax scale * log2(e)
};

// The three codes of 32 elements, and their scales, one a byte.
__device__ inline uint32_t cut_query(const uint16_t *at, i32x6 (&code)[3]) {
  uint4 x[4];
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[k] = ((const uint4 *)at)[k];
    const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
  }
  // 7.5 = 1.875 * 2^2; the scales stay bytes, and what underflows is below 2^-100.  With an infinity or NaN every score is NaN.
  const int e = max((int)(top >> 7) - 129 + ((top & 0x7Fu) > 0x70u ? 1 : 0), -92);
  bf16x32 r = __builtin_bit_cast(bf16x32, x);
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const float s = __uint_as_float((uint32_t)(127 + e - 4 * i) << 23);
    const auto c = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(r, s);
    code[i] = __builtin_bit_cast(i32x6, c);
    if (i < 2) {  // what is left, exactly: 8 bits at most
      const f32x32 back = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(c, s);
#pragma unroll
      for (int k = 0; k < 32; ++k) r[k] = (__bf16)((float)r[k] - back[k]);
    }
  }
  const uint32_t b = (uint32_t)(127 + e);
  return top >= 0x7F80u ? 0x00FFFFFFu : b | (b - 4) << 8 | (b - 8) << 16;
}

template <int A_BYTE, int PART>
__device__ inline f32x16 score_product(const uint4 k, const i32x6 (&q)[3], f32x16 acc, uint32_t k_scale, uint32_t q_scale) {
  const i32x8 a = {(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0};
  const i32x8 b = {q[PART][0], q[PART][1], q[PART][2], q[PART][3], q[PART][4], q[PART][5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, acc, 4, 2, A_BYTE, (int)k_scale, PART, (int)q_scale);
}

// The groups of V of a key that are NaN, for a row that sees it.
__device__ inline void put_nan(uint32_t bad, bool sees, f32x16 (&o)[4]) {
  if (bad == 0u) return;
#pragma unroll
  for (int db = 0; db < 4; ++db)
    if ((bad >> db & 1u) != 0u && sees)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] = NAN;
}

// 32 query rows a workgroup, every wave its own keys, tiles of 32 of them; no barriers on the way.  A lane reads the half row of K
// that it multiplies itself.
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
  // KV heads side by side, then splits, then row tiles from the longest down
  const int kvh = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv, sp = rest % p.S, r0 = (p.tiles - 1 - rest / p.S) * kRowsFew;
  const int seen_all = p.pos + r0 / p.g;     // last key that every row sees
  const int t_masked = (seen_all + 1) / KT;  // first tile that some do not
  const int n_tiles = (p.pos + (min(r0 + kRowsFew, p.rows) - 1) / p.g) / KT + 1;
  const int per = (n_tiles + p.S - 1) / p.S;
  const int t_begin = min(sp * per, n_tiles), t_end = min(t_begin + per, n_tiles);

  // this lane's row, and the last key that it sees
  const int row = min(r0 + q, p.rows - 1), tok = row / p.g, head = kvh * p.g + (row - tok * p.g), see = p.pos + tok;

  const size_t first = (size_t)kvh * p.capacity;
  const uint8_t *__restrict__ Kh = p.K + first * kRow4 + 32 * gg, *__restrict__ Vh = p.V + first * kRow4 + 16 * (lane & 3);
  const uint32_t *__restrict__ ksh = p.k_scale + first, *__restrict__ vsh = p.v_scale + first;

  uint4 kc[2], vc[2];  // a lane's two groups of K; pieces of V: rows lane / 4 and 16 further, a group each
  uint32_t ks, vs[2];
  auto fetch = [&](int t) {  // behind the tokens the last one again: nobody sees it there
    const size_t kr = min(t * KT + q, p.tokens - 1);
    kc[0] = *(const uint4 *)(Kh + kr * kRow4);
    kc[1] = *(const uint4 *)(Kh + kr * kRow4 + 16);
    ks = ksh[kr];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const size_t vr = min(t * KT + (lane >> 2) + 16 * i, p.tokens - 1);
      vc[i] = *(const uint4 *)(Vh + vr * kRow4);
      vs[i] = vsh[vr];
    }
  };
  int t = t_begin + wave;
  if (t < t_end) fetch(t);

  // Q: the groups 2gg and 2gg + 1 of a row, as the lane's K
  i32x6 qc[2][3];
  uint32_t qs[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) qs[s] = cut_query(p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs + 64 * gg + 32 * s, qc[s]);

  f32x16 oacc[4];
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  float m_run = -INFINITY;
  f32x4 lacc[2] = {};

  unsigned vbase;
  {
    const int r = lane & 15, part = (lane >> 4) & 1, vrow = 4 * gg + (r >> 2);
    vbase = (unsigned)(vrow * 256) | (unsigned)(((2 * part + ((r & 3) >> 1)) ^ ((vrow & 3) * 5)) << 4) | (unsigned)((r & 1) << 3);
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
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float s = scale4(vs[i] >> (8 * (lane & 3)) & 0xFFu);
      const uint32_t w[4] = {vc[i].x, vc[i].y, vc[i].z, vc[i].w};
      const int r = (lane >> 2) + 16 * i;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        *(uint4 *)((char *)lds.v[wave] + r * 256 + (((4 * (lane & 3) + k) ^ ((r & 3) * 5)) << 4)) = decode4_8(w[k], s);
    }
    const uint32_t ksw = ks >> (16 * gg);
    f32x16 sacc[1] = {};  // S^T = K Q^T
    sacc[0] = score_product<0, 0>(kc[0], qc[0], sacc[0], ksw, qs[0]);
    sacc[0] = score_product<0, 1>(kc[0], qc[0], sacc[0], ksw, qs[0]);
    sacc[0] = score_product<0, 2>(kc[0], qc[0], sacc[0], ksw, qs[0]);
    sacc[0] = score_product<1, 0>(kc[1], qc[1], sacc[0], ksw, qs[1]);
    sacc[0] = score_product<1, 1>(kc[1], qc[1], sacc[0], ksw, qs[1]);
    sacc[0] = score_product<1, 2>(kc[1], qc[1], sacc[0], ksw, qs[1]);
    if (t + WK < t_end) fetch(t + WK);
    wave_lds_sync();
    absorb_tile<PARTS>(sacc, (t + 1) * KT - 1 > seen_all, see - t * KT - 4 * gg, lds.v[wave], vbase, p.c, m_run, lacc, oacc);
    wave_lds_sync();
  }
  if (t_end > t_masked) {
    __syncthreads();
    for (int t = max(t_begin, t_masked); t < t_end; ++t) {
      if ((t - t_begin) % WK != wave) continue;  // another wave's tile
      for (int j = t * KT; j < (t + 1) * KT; ++j) put_nan(rowbad[j - t_masked * KT], j <= see, oacc);
    }
  }
  const float l_run = sum_pair(lacc[0][0] + lacc[1][0]);  // the keys of both lanes of a row
  put_waves(p, kvh, r0, sp, m_run, l_run, oacc, &lds.o[0][0][0], s_m, s_l);
}

// Many rows: four waves of 32 query rows each, which share tiles of 64 keys.  K goes from memory into LDS as it is (the LDS DMA, no registers), V
// in bf16, from registers that were read a tile ahead; beside the products of a tile, V of the next one.
__global__ __launch_bounds__(kThreads, 2) void attend4_rows_kernel(Attend4Args p) {
  constexpr int KT = 64;
  constexpr int kMasked = 3;  // tiles that some rows see and others do not, at most: 127 keys
  __shared__ __attribute__((aligned(16))) uint8_t Ks[2][KT * kRow4];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[2][KT * 128];
  __shared__ uint8_t rowbad[kMasked * KT];  // keys of the masked tiles: a bit for each group of V that is NaN

  const int tid = threadIdx.x, lane = tid & 63, q = lane & 31, gg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // KV heads side by side (workgroups go to the XCDs in turn: with 8 KV heads each stays in one L2), then splits, then row tiles
  const int kvh = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv, sp = rest % p.S, down = rest / p.S;
  const int rt = down < p.turn ? p.tiles - 1 - down : down - p.turn;
  const int r0 = rt * kRowsMany, r_last = min(r0 + kRowsMany, p.rows) - 1;
  const int seen_all = p.pos + r0 / p.g;                // last key that every row of the workgroup sees
  const int t_masked = (seen_all + 1) / KT;             // first tile that some do not
  const int n_tiles = (p.pos + r_last / p.g) / KT + 1;  // tiles that some row sees
  const int per = (n_tiles + p.S - 1) / p.S;
  const int t_begin = min(sp * per, n_tiles), t_end = min(t_begin + per, n_tiles);

  // this lane's row, and the last keys that it, its wave's first and its wave's last row see
  const int wr0 = min(r0 + 32 * wave, p.rows - 1), wr1 = min(r0 + 32 * wave + 31, p.rows - 1);
  const int row = min(r0 + 32 * wave + q, p.rows - 1), tok = row / p.g, head = kvh * p.g + (row - tok * p.g);
  const int see = p.pos + tok, see0 = p.pos + wr0 / p.g, see1 = p.pos + wr1 / p.g;

  const size_t first = (size_t)kvh * p.capacity;
  const uint8_t *__restrict__ Kh = p.K + first * kRow4, *__restrict__ Vh = p.V + first * kRow4;
  const uint32_t *__restrict__ ksh = p.k_scale + first, *__restrict__ vsh = p.v_scale + first;

  // ---- K: 64 rows of 64 bytes, the 16-byte chunk c of row r in place c ^ (r / 4) % 4, so that b128 reads of 16 rows hit 64 banks (the
  // lane that owns place x of row r reads chunk x ^ (r / 4) % 4).  Behind the tokens the last row again, here and below: nobody sees it there.
  const unsigned ldsK = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)&Ks[0][0] + wave * 1024;
  const int krow = 16 * wave + (lane >> 2), kch = ((lane & 3) ^ (lane >> 4)) << 4;
  auto issue_k = [&](int t, int buf) {
    const unsigned at = (unsigned)(min(krow, p.tokens - 1 - t * KT) * kRow4 + kch);
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(at), "s"(Kh + (size_t)t * KT * kRow4),
                 "s"(ldsK + (unsigned)(buf * KT * kRow4)) : "memory");
  };
  uint32_t ks[2];  // of the keys q and q + 32
  auto fetch_ks = [&](int t) {
    const uint32_t *at = ksh + (size_t)t * KT;
    const int lim = p.tokens - 1 - t * KT;
    ks[0] = at[min(q, lim)];
    ks[1] = at[min(q + 32, lim)];
  };
  // ---- V: a thread's group of 32 codes, row vrow
  uint4 vc;
  uint32_t vs;
  const int vrow = tid >> 2, vg = tid & 3;
  auto fetch_v = [&](int t) {
    const int r = min(vrow, p.tokens - 1 - t * KT);
    vc = *(const uint4 *)(Vh + (size_t)t * KT * kRow4 + (unsigned)(r * kRow4 + vg * 16));
    vs = vsh[(size_t)t * KT + (unsigned)r];
  };
  char *const vput = (char *)&Vs[0][0] + vrow * 256;
  const unsigned vswz = (unsigned)(4 * vg ^ (vrow & 3) * 5) << 4;
  // A row that does not see a key gives it weight 0, and 0 x NaN is not 0: in tiles that only some rows see, groups of V
  // that are NaN stay out of the products and come back at the end for the rows that do see them.
  auto screen = [&](int t) {
    const bool bad = (vs >> (8 * vg) & 0xFFu) == kNanScale;
    const uint64_t who = __ballot(bad);
    if (vg == 0) rowbad[(t - t_masked) * KT + vrow] = (uint8_t)(who >> lane & 15ull);
    if (bad) { vc = make_uint4(0u, 0u, 0u, 0u); vs = 0x7F7F7F7Fu; }
  };
  if (t_begin < t_end) {
    fetch_v(t_begin);
    issue_k(t_begin, 0);
    fetch_ks(t_begin);
  }

  i32x6 qc[2][3];
  uint32_t qs[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) qs[s] = cut_query(p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs + 64 * gg + 32 * s, qc[s]);

  f32x16 oacc[4];
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  float m_run = -INFINITY;
  f32x4 lacc[2] = {};
  unsigned vbase;
  {
    const int r = lane & 15, part = (lane >> 4) & 1, vr = 4 * gg + (r >> 2);
    vbase = (unsigned)(vr * 256) | (unsigned)(((2 * part + ((r & 3) >> 1)) ^ ((vr & 3) * 5)) << 4) | (unsigned)((r & 1) << 3);
  }
  const unsigned kbase = (unsigned)(q * kRow4) | (unsigned)(((2 * gg) ^ (q >> 2 & 3)) << 4);

  if (t_begin < t_end) {
    if (t_begin >= t_masked) screen(t_begin);
    const float s = scale4(vs >> (8 * vg) & 0xFFu);
    const uint32_t w[4] = {vc.x, vc.y, vc.z, vc.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) *(uint4 *)(vput + (vswz ^ (unsigned)(k << 4))) = decode4_8(w[k], s);
    if (t_begin + 1 < t_end) fetch_v(t_begin + 1);
  }
  for (int t = t_begin; t < t_end; ++t) {
    const int cur = (t - t_begin) & 1, j0 = t * KT;
    // K of this tile has landed, and V of the next one; after the barrier both buffers of the tile hold it and
    // every wave is done with the tile before
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    __syncthreads();
    const uint32_t ksw[2] = {ks[0] >> (16 * gg), ks[1] >> (16 * gg)};
    if (t + 1 < t_end) {
      issue_k(t + 1, cur ^ 1);
      fetch_ks(t + 1);
      if (t + 1 >= t_masked) screen(t + 1);
    }
    // S^T = K Q^T, three products per fragment of K; beside them V of the next tile becomes bf16 (what is left in the
    // registers, behind the last tile: nobody reads it)
    const char *Kt = (const char *)&Ks[cur][0];
    uint4 kf[2][2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) kf[s][hf] = *(const uint4 *)(Kt + (kbase ^ (unsigned)(s << 4)) + hf * 32 * kRow4);
    f32x16 sacc[2] = {};
    const float vscale = scale4(vs >> (8 * vg) & 0xFFu);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sacc[0] = i == 0 ? score_product<0, 0>(kf[0][0], qc[0], sacc[0], ksw[0], qs[0]) : i == 1 ? score_product<0, 2>(kf[0][0], qc[0], sacc[0], ksw[0], qs[0])
              : i == 2 ? score_product<1, 0>(kf[1][0], qc[1], sacc[0], ksw[0], qs[1]) : score_product<1, 2>(kf[1][0], qc[1], sacc[0], ksw[0], qs[1]);
      sacc[1] = i == 0 ? score_product<0, 0>(kf[0][1], qc[0], sacc[1], ksw[1], qs[0]) : i == 1 ? score_product<0, 2>(kf[0][1], qc[0], sacc[1], ksw[1], qs[0])
              : i == 2 ? score_product<1, 0>(kf[1][1], qc[1], sacc[1], ksw[1], qs[1]) : score_product<1, 2>(kf[1][1], qc[1], sacc[1], ksw[1], qs[1]);
      if ((i & 1) == 0) {
        sacc[0] = i == 0 ? score_product<0, 1>(kf[0][0], qc[0], sacc[0], ksw[0], qs[0]) : score_product<1, 1>(kf[1][0], qc[1], sacc[0], ksw[0], qs[1]);
        sacc[1] = i == 0 ? score_product<0, 1>(kf[0][1], qc[0], sacc[1], ksw[1], qs[0]) : score_product<1, 1>(kf[1][1], qc[1], sacc[1], ksw[1], qs[1]);
      }
      const uint32_t w = i == 0 ? vc.x : i == 1 ? vc.y : i == 2 ? vc.z : vc.w;
      *(uint4 *)(vput + (cur ^ 1) * KT * 256 + (vswz ^ (unsigned)(i << 4))) = decode4_8(w, vscale);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (t + 2 < t_end) fetch_v(t + 2);
    if (j0 <= see1) absorb_tile<1>(sacc, j0 + KT - 1 > see0, see - j0 - 4 * gg, Vs[cur], vbase, p.c, m_run, lacc, oacc);
  }
  if (t_end > t_masked) {
    __syncthreads();
    for (int j = max(t_begin, t_masked) * KT; j < t_end * KT; ++j) put_nan(rowbad[j - t_masked * KT], j <= see, oacc);
  }
  const float l_run = sum_pair(lacc[0][0] + lacc[1][0]);  // the keys of both lanes of a row
  if (r0 + 32 * wave + q < p.rows) put_row(p, kvh, row, head, tok, sp, gg, m_run, l_run, oacc);
}

// Rows x splits that the scratch holds: two workgroups of 128 rows a compute unit, as for the 8-bit cache.
size_t max_slots(const Shape &sh) { return (size_t)sh.n_cu * 256; }

// Splits: as many as give two workgroups a compute unit.
struct Plan { bool few; int S; };
Plan plan_of(const Shape &sh, int rows, int tokens) {
  const bool few = rows <= 64;
  const int per = few ? kRowsFew : kRowsMany, keys = few ? 32 : 64;
  const int64_t wgs = (rows + per - 1) / per * (int64_t)sh.Hkv, all = (int64_t)rows * sh.Hkv;
  const int tiles = (tokens + keys - 1) / keys;
  const int64_t top = std::min<int64_t>(std::min(tiles / 4 + 1, kMaxSplits), (int64_t)max_slots(sh) / all);
  const int S = (int)std::max<int64_t>(1, std::min<int64_t>(2 * sh.n_cu / wgs, top)), share = (tiles + S - 1) / S;
  return {few, (tiles + share - 1) / share};
}

}  // namespace

void cache4_attend_plan(const Shape &sh, int n, int pos, int *rows, int *splits) {
  const Plan plan = plan_of(sh, sh.g * n, pos + n);
  *rows = plan.few ? kRowsFew : kRowsMany;
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
  const Plan plan = plan_of(sh, a.rows, a.tokens);
  a.S = plan.S;
  a.tiles = (a.rows + (plan.few ? kRowsFew : kRowsMany) - 1) / (plan.few ? kRowsFew : kRowsMany);
  const int64_t wgs = (int64_t)a.tiles * sh.Hkv;
  a.turn = a.tiles;
  if (!plan.few && wgs * a.S > sh.n_cu && wgs * a.S <= 2 * sh.n_cu) a.turn = std::max(1, (int)(sh.n_cu / (sh.Hkv * a.S)));
  const int64_t all = (int64_t)a.rows * sh.Hkv;
  a.ml = (float2 *)scratch;
  a.part = (float *)((char *)scratch + max_slots(sh) * 8);
  const unsigned grid = (unsigned)(wgs * a.S);
  if (plan.few && a.rows <= 2 * kRowsFew) attend4_few_kernel<2><<<grid, kThreads, 0, st>>>(a);
  else if (plan.few) attend4_few_kernel<1><<<grid, kThreads, 0, st>>>(a);
  else attend4_rows_kernel<<<grid, kThreads, 0, st>>>(a);
  launch_join(a, all, st);
  return hipGetLastError();
}

}  // namespace sa
