// Causal attention of the newest n tokens over the 8-bit cache: O = softmax(scale Q K^T) V, row by row, with the running
// maximum and sum of an online softmax, for n from one token to thousands.
//
// The g query heads of a KV head read the same keys, so its g n query rows (token, head of the group) are taken
// together, 32 to a wave: a decode step of 8 heads a group fills 8 rows of one wave's products, a chunk of a prompt
// fills workgroups of 128 rows.  The tile step is that of the sparse prefill: S^T = K Q^T, so that a lane owns a query row,
// and O^T += V^T P^T in v_mfma_f32_32x32x16_bf16 with transposing LDS reads.  Two shapes of a workgroup (4 waves):
//   few rows   32 rows, each wave every fourth tile of 32 keys, in LDS of its own, no barriers.  Bound: memory; one token
//              of 32 heads at 128K keys (270 MB) 53.5 us, 5.0 TB/s
//   many rows  each wave 32 of 128 rows, tiles of 64 keys shared by the four, K in codes for the 8-bit products.  Bound: matrix
//              pipe, busy 65 % of the time, at the 2.0 GHz that the power limit leaves: 2048 tokens at 64K keys 1.70 to 1.79 ms
//              with the card, 1.27 PFLOP/s, where a large bf16 product of the library reaches 1.32
// and the keys are split over workgroups where rows alone do not fill the card; the splits' sums are joined by a second
// launch (plan_of, at the end, says which shape and how many splits).
#include <algorithm>
#include <cmath>

#include "attend_common.h"
#include "cache_codes.h"
#include "sa_internal.h"

namespace sa {
namespace {

constexpr int kRowsMany = 128, kRowsFew = 32;  // query rows of a workgroup

struct AttendArgs : AttendOut {
  const uint16_t *Q;
  const uint8_t *K, *V;
  const float *k_scale, *v_scale;
  const uint16_t *k_open, *v_open;
  int64_t q_hs, q_rs, capacity;
  int tiles;                   // row tiles
  int turn;                    // many rows: row tiles from the last one down, this many, then from the first one up; few: the first one
                               // of those that go down, or 0
  int shift;                   // log2 of the block
  int pos, tokens, closed;     // of the first query; in the cache; in its full blocks
  float c;                     // softmax scale * log2(e)
};

// 16 codes of a row, 8 words of bf16.
template <int TYPE>
__device__ inline void decode16(const uint4 x, float scale, uint4 &lo, uint4 &hi) {
  lo.x = decode2<TYPE, false>(x.x, scale); lo.y = decode2<TYPE, true>(x.x, scale);
  lo.z = decode2<TYPE, false>(x.y, scale); lo.w = decode2<TYPE, true>(x.y, scale);
  hi.x = decode2<TYPE, false>(x.z, scale); hi.y = decode2<TYPE, true>(x.z, scale);
  hi.z = decode2<TYPE, false>(x.w, scale); hi.w = decode2<TYPE, true>(x.w, scale);
}

// Whether a pair of bf16 values holds an infinity or NaN; and the pair without it.
__device__ inline uint32_t nonfinite(uint32_t w) { return ((w & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u; }
__device__ inline uint32_t finite_only(uint32_t w) {
  const uint32_t bad = nonfinite(w);
  return w & ~((bad << 1) - (bad >> 15));
}

// Element d of key j of K or V, as the cache has it.
template <int TYPE>
__device__ inline float element(const AttendArgs &p, int kvh, const uint8_t *codes, const float *scale, const uint16_t *open, int j, int d) {
  if (j >= p.closed) return value(open[(((size_t)kvh << p.shift) + (j - p.closed)) * kHeadDim + d]);
  return decode2f<TYPE, false>(codes[((size_t)kvh * p.capacity + j) * kHeadDim + d])[0] * scale[(size_t)kvh * (p.capacity >> p.shift) + (j >> p.shift)];
}

// The non-finite values of V of key j, which the products have been kept from, added for a lane's row if it sees the key.
// Seldom there, so the score is taken once more, plainly.
template <int TYPE>
__device__ inline void add_nonfinite(const AttendArgs &p, int kvh, int j, int head, int tok, int see, int gg, float m, f32x16 (&o)[4]) {
  float s = 0.f;
  for (int d = 0; d < kHeadDim; ++d)
    s = __builtin_fmaf(value(p.Q[(size_t)head * p.q_hs + (size_t)tok * p.q_rs + d]), element<TYPE>(p, kvh, p.K, p.k_scale, p.k_open, j, d), s);
  const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s, p.c, m == -INFINITY ? 0.f : -m));
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float v = element<TYPE>(p, kvh, p.V, p.v_scale, p.v_open, j, 32 * db + 8 * (r / 4) + 4 * gg + r % 4);
      if (j <= see && !__builtin_isfinite(v)) o[db][r] += w * v;
      __builtin_amdgcn_sched_barrier(0);
    }
}

// Few rows: 32 query rows a workgroup, every wave its own keys, tiles of 32 of them; no barriers on the way.  A lane reads half a row
// of K, which it multiplies itself (the order of the elements of a product is free, Q has the same), and turns it into bf16 between the
// products.  V becomes bf16 on its way into LDS, for the transposing reads.  Both are read a tile ahead.  (With K through LDS too, 250
// tokens of 32 heads at 2200 keys took 27.8 us instead of 19.0, one at 128K 53.8 instead of 52.0.)
template <int TYPE, int PARTS>
__global__ __launch_bounds__(kThreads, 2) void attend_few_kernel(AttendArgs p) {
  constexpr int KT = 32, WK = kThreads / 64;  // keys per tile, waves
  constexpr int NC = KT * 8 / 64;             // 16-byte pieces of codes of K, and of V, that a lane reads per tile
  constexpr int kMasked = 2;                  // tiles that some rows see and others do not, at most: 31 keys
  __shared__ __attribute__((aligned(16))) union {
    uint16_t v[WK][KT * 128];
    float o[WK][32][kHeadDim];
  } lds;
  __shared__ uint8_t rowbad[kMasked * KT];  // keys of the masked tiles whose V has an infinity or NaN
  __shared__ float s_m[4][32], s_l[4][32];

  const int tid = threadIdx.x, lane = tid & 63, q = lane & 31, gg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // KV heads side by side, then splits, then row tiles
  const int kvh = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv, sp = rest % p.S, r0 = abs(p.turn - rest / p.S) * kRowsFew;
  const int seen_all = p.pos + r0 / p.g;     // last key that every row sees
  const int t_masked = (seen_all + 1) / KT;  // first tile that some do not
  const int n_tiles = (p.pos + (min(r0 + kRowsFew, p.rows) - 1) / p.g) / KT + 1;
  const int per = (n_tiles + p.S - 1) / p.S;
  const int t_begin = min(sp * per, n_tiles), t_end = min(t_begin + per, n_tiles);
  const int t_full = min(t_end, p.closed / KT);  // tiles t_begin .. t_full - 1 are codes

  // this lane's row, and the last key that it sees
  const int row = min(r0 + q, p.rows - 1), tok = row / p.g, head = kvh * p.g + (row - tok * p.g), see = p.pos + tok;

  const uint8_t *__restrict__ Kh = p.K + (size_t)kvh * p.capacity * kHeadDim + q * kHeadDim + 64 * gg;
  const uint8_t *__restrict__ Vh = p.V + (size_t)kvh * p.capacity * kHeadDim + lane * 16;
  const float *ksh = p.k_scale + (size_t)kvh * (p.capacity >> p.shift), *vsh = p.v_scale + (size_t)kvh * (p.capacity >> p.shift);

  uint4 kc[NC], vc[NC];
  float ksc = 1.f, vsc = 1.f;
  auto fetch = [&](int t) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      kc[i] = *(const uint4 *)(Kh + (size_t)t * KT * kHeadDim + 16 * i);
      vc[i] = *(const uint4 *)(Vh + (size_t)t * KT * kHeadDim + 1024 * i);
    }
    ksc = ksh[(t * KT) >> p.shift];
    vsc = vsh[(t * KT) >> p.shift];
  };
  // A wave's tiles of codes are t_first and every fourth one, from a place on that puts the splits 512 KB / S apart modulo 512 KB:
  // at the same distance of, say, 256 KB all of them ask the same few memory channels at a time (from the first tile on: one token at
  // 130000 keys 60.3 us instead of 53.2, 16 tokens 84.9 instead of 67.6).
  const int t_first = t_begin + wave, mine = max(0, (t_full - t_first + WK - 1) / WK);
  int t = t_first;
  if (mine > 0) t += ((sp * 128 / p.S - t_begin & 127) / WK) % mine * WK;
  if (mine > 0) fetch(t);

  bf16x8 qf[8];  // Q^T fragments: B operand, lane = query row, 8 consecutive d of the lane's half
  {
    const uint16_t *qrow = p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const bf16x8 *)(qrow + 64 * gg + 8 * ks);
  }
  f32x16 oacc[4];
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  float m_run = -INFINITY;
  f32x4 lacc[2] = {};

  // LDS tiles are KT rows x 256 B, the 16-byte chunk c of row r at c ^ ((r & 3) << 2): transposing b64 reads hit 64 banks.
  unsigned vbase;
  {
    const int r = lane & 15, part = (lane >> 4) & 1, vrow = 4 * gg + (r >> 2);
    vbase = (unsigned)(vrow * 256) | (unsigned)(((2 * part + ((r & 3) >> 1)) ^ ((vrow & 3) << 2)) << 4) | (unsigned)((r & 1) << 3);
  }
  auto put_v = [&](int i, int half, const uint4 &x) {  // 8 elements of piece i
    const int r = (lane >> 3) + 8 * i, c = 2 * (lane & 7) + half;
    *(uint4 *)((char *)lds.v[wave] + r * 256 + ((c ^ ((r & 3) << 2)) << 4)) = x;
  };
  // A row that does not see a key gives it weight 0, and 0 x inf is not 0: in tiles that only some rows see, non-finite values
  // of V stay out of the products and come back at the end for the rows that do see them.
  auto mark = [&](int t, int i, bool bad) {
    const uint64_t who = __ballot(bad);
    if ((lane & 7) == 0) rowbad[(t - t_masked) * KT + (lane >> 3) + 8 * i] = ((who >> (lane & 56)) & 0xFFull) != 0ull;
    return who != 0ull;
  };
  auto absorb = [&](int t, f32x16 (&sacc)[1]) {
    wave_lds_sync();
    absorb_tile<PARTS>(sacc, (t + 1) * KT - 1 > seen_all, see - t * KT - 4 * gg, lds.v[wave], vbase, p.c, m_run, lacc, oacc);
    wave_lds_sync();
  };
  for (int left = mine; left > 0; --left) {
    if (t >= t_masked) {
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (mark(t, i, (nonfinite_codes<TYPE>(vc[i].x) | nonfinite_codes<TYPE>(vc[i].y) | nonfinite_codes<TYPE>(vc[i].z) | nonfinite_codes<TYPE>(vc[i].w)) != 0u))
          vc[i] = make_uint4(finite_codes<TYPE>(vc[i].x), finite_codes<TYPE>(vc[i].y), finite_codes<TYPE>(vc[i].z), finite_codes<TYPE>(vc[i].w));
    }
    f32x16 sacc[1];  // S^T = K Q^T
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // beside the products, V into LDS
      auto words = [&](const uint4 &x, float scale) {
        const uint32_t c0 = i & 1 ? x.z : x.x, c1 = i & 1 ? x.w : x.y;
        return make_uint4(decode2<TYPE, false>(c0, scale), decode2<TYPE, true>(c0, scale), decode2<TYPE, false>(c1, scale), decode2<TYPE, true>(c1, scale));
      };
      const f32x16 zero = {};
      const uint4 kf = words(kc[i >> 1], ksc);
      const u32x4 kv = {kf.x, kf.y, kf.z, kf.w};
      sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kv), qf[i], i == 0 ? zero : sacc[0], 0, 0, 0);
      put_v(i >> 1, i & 1, words(vc[i >> 1], vsc));
      __builtin_amdgcn_sched_barrier(0);
    }
    const int now = t;
    t = t + WK < t_full ? t + WK : t_first;
    if (left > 1) fetch(t);
    absorb(now, sacc);
  }
  // the open block: bf16 rows; behind the tokens the last one again, and zeros for V
  for (t = t_first + mine * WK; t < t_end; t += WK) {
    const size_t first = (size_t)kvh << p.shift;
    const uint16_t *krow = p.k_open + (first + (size_t)(min(t * KT + q, p.tokens - 1) - p.closed)) * kHeadDim + 64 * gg;
    bf16x8 kf[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) kf[i] = *(const bf16x8 *)(krow + 8 * i);
    uint4 lo[NC], hi[NC];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const size_t at = (first + (size_t)(min(t * KT + (lane >> 3) + 8 * i, p.tokens - 1) - p.closed)) * kHeadDim + (lane & 7) * 16;
      lo[i] = *(const uint4 *)(p.v_open + at);
      hi[i] = *(const uint4 *)(p.v_open + at + 8);
    }
    f32x16 sacc[1] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) sacc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], qf[i], sacc[0], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (t * KT + (lane >> 3) + 8 * i >= p.tokens) lo[i] = hi[i] = make_uint4(0u, 0u, 0u, 0u);
      if (t >= t_masked &&
          mark(t, i, (nonfinite(lo[i].x) | nonfinite(lo[i].y) | nonfinite(lo[i].z) | nonfinite(lo[i].w) |
                      nonfinite(hi[i].x) | nonfinite(hi[i].y) | nonfinite(hi[i].z) | nonfinite(hi[i].w)) != 0u)) {
        lo[i] = make_uint4(finite_only(lo[i].x), finite_only(lo[i].y), finite_only(lo[i].z), finite_only(lo[i].w));
        hi[i] = make_uint4(finite_only(hi[i].x), finite_only(hi[i].y), finite_only(hi[i].z), finite_only(hi[i].w));
      }
      put_v(i, 0, lo[i]);
      put_v(i, 1, hi[i]);
    }
    absorb(t, sacc);
  }
  // Non-finite values of V in tiles that only some rows see: their share, for the rows that do.  Seldom there, so the
  // scores are taken once more, plainly.
  if (t_end > t_masked) {
    __syncthreads();
    for (int t = max(t_begin, t_masked); t < t_end; ++t) {
      if ((t - t_begin) % WK != wave) continue;  // another wave's tile
      for (uint64_t bad = __ballot(lane < KT && rowbad[(t - t_masked) * KT + (lane & (KT - 1))] != 0); bad != 0ull; bad &= bad - 1ull)
        add_nonfinite<TYPE>(p, kvh, t * KT + __ffsll((unsigned long long)bad) - 1, head, tok, see, gg, m_run, oacc);
    }
  }
  const float l_run = sum_pair(lacc[0][0] + lacc[1][0]);  // the keys of both lanes of a row

  put_waves(p, kvh, r0, sp, m_run, l_run, oacc, &lds.o[0][0][0], s_m, s_l);
}

// Many rows: four waves of 32 query rows each, which share tiles of 64 keys.
//   K stays in codes: they go from memory into LDS as they are (the LDS DMA, no registers) and into the 8-bit matrix
//   instructions, at twice the rate of the bf16 ones.  Q, in bf16, is cut into two codes of e4m3, q = hi + lo: hi is q
//   rounded to 4 significant bits, and what is left fits 4 more, exactly, so that two products at twice the rate
//   multiply all of q.  (The largest element of a row, if 2^-92 or more, lies in (224, 448] scales; one below 2^-6 scales is rounded to a
//   16th of the least code: off by 2^-14 scales, 2^-21.8 of the row's largest, at most.)  The scales of Q's rows and of the block of K are
//   exponents that the instruction takes.
//   V has to be multiplied with probabilities, which need bf16: its codes are turned into bf16 on their way into LDS, from
//   registers that were read a tile ahead.
template <int TYPE>
__global__ __launch_bounds__(kThreads, 2) void attend_rows_kernel(AttendArgs p) {
  constexpr int KT = 64, T = kThreads, NC = KT * 8 / T;  // NC: 16-byte pieces of K, and of V, that a thread moves per tile
  constexpr int kMasked = 3;                             // tiles that some rows see and others do not, at most: 127 keys
  // K of two tiles as codes, or of one in bf16 (open block); V of two tiles in bf16
  __shared__ __attribute__((aligned(16))) uint8_t Ks[2][KT * 128];
  __shared__ __attribute__((aligned(16))) uint16_t Vs[2][KT * 128];
  __shared__ uint8_t rowbad[kMasked * KT];  // keys of the masked tiles whose V has an infinity or NaN

  const int tid = threadIdx.x, lane = tid & 63, q = lane & 31, gg = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // KV heads side by side (workgroups go to the XCDs in turn: with 8 KV heads each stays in one L2), then splits, then row tiles
  const int kvh = blockIdx.x % p.Hkv, rest = blockIdx.x / p.Hkv, sp = rest % p.S, down = rest / p.S;
  const int rt = down < p.turn ? p.tiles - 1 - down : down - p.turn;
  const int r0 = rt * kRowsMany, r_last = min(r0 + kRowsMany, p.rows) - 1;
  const int seen_all = p.pos + r0 / p.g;                 // last key that every row of the workgroup sees
  const int t_masked = (seen_all + 1) / KT;              // first tile that some do not
  const int n_tiles = (p.pos + r_last / p.g) / KT + 1;   // tiles that some row sees
  const int per = (n_tiles + p.S - 1) / p.S;
  const int t_begin = min(sp * per, n_tiles), t_end = min(t_begin + per, n_tiles);
  const int n_closed = p.closed / KT, t_full = min(t_end, n_closed);  // tiles t_begin .. t_full - 1 are codes

  // this lane's row, and the last keys that it, its wave's first and its wave's last row see
  const int wr0 = min(r0 + 32 * wave, p.rows - 1), wr1 = min(r0 + 32 * wave + 31, p.rows - 1);
  const int row = min(r0 + 32 * wave + q, p.rows - 1), tok = row / p.g, head = kvh * p.g + (row - tok * p.g);
  const int see = p.pos + tok, see0 = p.pos + wr0 / p.g, see1 = p.pos + wr1 / p.g;

  const uint8_t *__restrict__ Kh = p.K + (size_t)kvh * p.capacity * kHeadDim;
  const uint8_t *__restrict__ Vh = p.V + (size_t)kvh * p.capacity * kHeadDim;
  const float *ksh = p.k_scale + (size_t)kvh * (p.capacity >> p.shift), *vsh = p.v_scale + (size_t)kvh * (p.capacity >> p.shift);

  // ---- K: 64 rows of 128 bytes, the 16-byte chunks of row r XOR-swizzled by r / 2 (the swizzle is applied on the global
  // side: the lane that owns chunk c of row r reads chunk c ^ (r / 2) % 8), so that b128 reads of 8 rows hit 64 banks.
  const unsigned ldsK = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)&Ks[0][0] + wave * 1024;
  const unsigned kvoff = (unsigned)((8 * wave + (lane >> 3)) * 128 + (((lane & 7) ^ ((lane >> 4) | (wave & 1) << 2)) << 4));
  auto issue_k = [&](int t, int buf) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const uint8_t *src = Kh + ((size_t)t * KT + 32 * i) * kHeadDim;
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(kvoff), "s"(src),
                   "s"(ldsK + (unsigned)(buf * KT * 128 + i * T * 16)) : "memory");
    }
  };
  // ---- V: a thread's pieces of 16 codes, row vrow + 32 i
  uint4 vc[NC];
  const int vrow = tid >> 3, vch = tid & 7;
  auto fetch_v = [&](int t) {
#pragma unroll
    for (int i = 0; i < NC; ++i) vc[i] = *(const uint4 *)(Vh + (size_t)t * KT * kHeadDim + tid * 16 + i * T * 16);
  };
  auto put_v = [&](int buf, int i, const uint4 &lo, const uint4 &hi) {
    char *at = (char *)&Vs[buf][0] + (vrow + 32 * i) * 256;
    const int swz = (vrow & 3) << 2;
    *(uint4 *)(at + (((2 * vch) ^ swz) << 4)) = lo;
    *(uint4 *)(at + (((2 * vch + 1) ^ swz) << 4)) = hi;
  };
  // Non-finite values of V in a tile that only some rows see: a row that does not gives them weight 0, and 0 x inf is not
  // 0.  They stay out of the products and come back at the end for the rows that do.
  auto mark = [&](int t, int i, bool bad) {
    const uint64_t who = __ballot(bad);
    if (vch == 0) rowbad[(t - t_masked) * KT + vrow + 32 * i] = ((who >> (lane & 56)) & 0xFFull) != 0ull;
  };
  auto screen = [&](int t) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      mark(t, i, (nonfinite_codes<TYPE>(vc[i].x) | nonfinite_codes<TYPE>(vc[i].y) | nonfinite_codes<TYPE>(vc[i].z) | nonfinite_codes<TYPE>(vc[i].w)) != 0u);
      vc[i] = make_uint4(finite_codes<TYPE>(vc[i].x), finite_codes<TYPE>(vc[i].y), finite_codes<TYPE>(vc[i].z), finite_codes<TYPE>(vc[i].w));
    }
  };

  const bool open = t_end > max(t_begin, n_closed);  // has tiles of the open block, which come first
  if (t_begin < t_full) {  // on their way while Q is read and cut
    fetch_v(t_begin);
    if (!open) issue_k(t_begin, 0);
  }
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
    vbase = (unsigned)(vr * 256) | (unsigned)(((2 * part + ((r & 3) >> 1)) ^ ((vr & 3) << 2)) << 4) | (unsigned)((r & 1) << 3);
  }

  // ---- tiles multiplied in bf16, with whole queries ---------------------------------------------------------
  auto whole_tiles = [&](int from) {
    if (from >= t_end) return;
    bf16x8 qf[8];  // Q^T fragments: B operand, lane = row, 8 consecutive d per k-step half
    const uint16_t *qrow = p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const bf16x8 *)(qrow + 16 * ks + 8 * gg);
    for (int t = from; t < t_end; ++t) {
      const int j0 = t * KT;
      uint16_t *const Kt = (uint16_t *)&Ks[0][0];  // both buffers
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int r = vrow + 32 * i, j = j0 + r;
        uint4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = make_uint4(0u, 0u, 0u, 0u);
        if (TYPE == SA_CACHE_E5M2 && j < p.closed) {
          const size_t at = (size_t)j * kHeadDim + vch * 16;
          decode16<TYPE>(*(const uint4 *)(Kh + at), ksh[j >> p.shift], x[0], x[1]);
          decode16<TYPE>(*(const uint4 *)(Vh + at), vsh[j >> p.shift], x[2], x[3]);
        } else if (j < p.tokens) {  // zeros behind the tokens
          const size_t at = (((size_t)kvh << p.shift) + (j - p.closed)) * kHeadDim + vch * 16;
          x[0] = *(const uint4 *)(p.k_open + at);
          x[1] = *(const uint4 *)(p.k_open + at + 8);
          x[2] = *(const uint4 *)(p.v_open + at);
          x[3] = *(const uint4 *)(p.v_open + at + 8);
        }
        if (t >= t_masked) {
          uint32_t bad = 0u;
#pragma unroll
          for (int k = 2; k < 4; ++k) {
            bad |= nonfinite(x[k].x) | nonfinite(x[k].y) | nonfinite(x[k].z) | nonfinite(x[k].w);
            x[k] = make_uint4(finite_only(x[k].x), finite_only(x[k].y), finite_only(x[k].z), finite_only(x[k].w));
          }
          mark(t, i, bad != 0u);
        }
        char *at = (char *)Kt + r * 256;  // chunk c of row r at c ^ (r & 15)
        *(uint4 *)(at + (((2 * vch) ^ (r & 15)) << 4)) = x[0];
        *(uint4 *)(at + (((2 * vch + 1) ^ (r & 15)) << 4)) = x[1];
        put_v(1, i, x[2], x[3]);
      }
      __syncthreads();
      if (j0 <= see1) {
        f32x16 sacc[2] = {};
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const bf16x8 kf = *(const bf16x8 *)((const char *)Kt + (32 * hf + q) * 256 + (((2 * ks + gg) ^ (q & 15)) << 4));
            sacc[hf] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], sacc[hf], 0, 0, 0);
          }
        absorb_tile<1>(sacc, j0 + KT - 1 > see0, see - j0 - 4 * gg, Vs[1], vbase, p.c, m_run, lacc, oacc);
      }
    }
  };
  whole_tiles(max(t_begin, n_closed));  // the open block first
  if (open && t_begin < t_full) {
    __syncthreads();
    issue_k(t_begin, 0);
  }

  if (t_begin < t_full) {
    // ---- Q in codes: scales 2^e (hi) and 2^(e - 4) (lo) of a row, the least e with every |q| <= 448 2^e
    i32x8 qc[2][2];  // [64 d][hi, lo]: bytes d = 64 s + 32 gg ..
    int qscale[2];
    {
      uint32_t top = 0;
      const uint16_t *qrow = p.Q + (size_t)head * p.q_hs + (size_t)tok * p.q_rs;
      uint4 x[2][4];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          x[s][k] = *(const uint4 *)(qrow + 64 * s + 32 * gg + 8 * k);
          const uint32_t w[4] = {x[s][k].x, x[s][k].y, x[s][k].z, x[s][k].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
        }
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      const int e = scale_exponent<SA_CACHE_E4M3>(min(top, 0x7F7Fu));
      const float up = __uint_as_float((uint32_t)(127 - e) << 23);
      qscale[0] = 127 + e;
      qscale[1] = 127 + e - 4;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t w[4] = {x[s][k].x, x[s][k].y, x[s][k].z, x[s][k].w};
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            const uint32_t hi = encode4<SA_CACHE_E4M3>(w[i], w[i + 1], up);
            const f32_pair h0 = decode2f<SA_CACHE_E4M3, false>(hi), h1 = decode2f<SA_CACHE_E4M3, true>(hi);
            const float l0 = (value((uint16_t)w[i]) * up - h0[0]) * 16.f, l1 = (value((uint16_t)(w[i] >> 16)) * up - h0[1]) * 16.f;
            const float l2 = (value((uint16_t)w[i + 1]) * up - h1[0]) * 16.f, l3 = (value((uint16_t)(w[i + 1] >> 16)) * up - h1[1]) * 16.f;
            int lo = __builtin_amdgcn_cvt_pk_fp8_f32(l0, l1, 0, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(l2, l3, lo, true);
            qc[s][0][2 * k + i / 2] = (int)hi;
            qc[s][1][2 * k + i / 2] = lo;
          }
        }
    }
    const unsigned kbase = (unsigned)(q * 128) | (unsigned)((((2 * gg) ^ (q >> 1)) & 7) << 4);
    constexpr int kType = TYPE == SA_CACHE_E4M3 ? 0 : 1;

    float vsc = uniform_load(vsh, (t_begin * KT) >> p.shift);
    auto convert_v = [&](int buf, int i) {
      uint4 lo, hi;
      decode16<TYPE>(vc[i], vsc, lo, hi);
      put_v(buf, i, lo, hi);
    };
    if (t_begin >= t_masked) screen(t_begin);
#pragma unroll
    for (int i = 0; i < NC; ++i) convert_v(0, i);
    if (t_begin + 1 < t_full) {
      fetch_v(t_begin + 1);
      vsc = uniform_load(vsh, ((t_begin + 1) * KT) >> p.shift);
    }
    for (int t = t_begin; t < t_full; ++t) {
      const int cur = (t - t_begin) & 1, j0 = t * KT;
      // K of this tile has landed, and V of the next one; after the barrier both buffers of the tile hold it and
      // every wave is done with the tile before
      __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
      __syncthreads();
      const bool more = t + 1 < t_full;
      if (more) {
        issue_k(t + 1, cur ^ 1);
        if (t + 1 >= t_masked) screen(t + 1);
      }
      // S^T = K Q^T, two products per fragment of K, the reads of the fragment after the next behind them; beside them V of
      // the next tile becomes bf16 (what is left in the registers, behind the last tile: nobody reads it)
      const int kscale = (int)(__float_as_uint(uniform_load(ksh, j0 >> p.shift)) >> 23);
      const char *Kt = (const char *)&Ks[cur][0];
      auto k_frag = [&](int f) {
        const unsigned at = (kbase ^ (unsigned)((f >> 1) << 6)) + (f & 1) * 32 * 128;
        return __builtin_shufflevector(*(const i32x4 *)(Kt + at), *(const i32x4 *)(Kt + (at ^ 16u)), 0, 1, 2, 3, 4, 5, 6, 7);
      };
      f32x16 sacc[2];
      i32x8 kf[2];
      uint4 vx[2];
      kf[0] = k_frag(0);
      kf[1] = k_frag(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int f = i >> 1, hf = f & 1, s = f >> 1, part = i & 1;
        const f32x16 zero = {};
        sacc[hf] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(kf[f & 1], qc[s][part], s == 0 && part == 0 ? zero : sacc[hf], kType, 0, 0, kscale,
                                                                  0, qscale[part]);
        if (part == 1 && f + 2 < 4) kf[f & 1] = k_frag(f + 2);
#pragma unroll
        for (int w = NC * i; w < NC * (i + 1); ++w) {
          const uint32_t code = w & 4 ? (w & 2 ? vc[w >> 3].w : vc[w >> 3].z) : (w & 2 ? vc[w >> 3].y : vc[w >> 3].x);
          const uint32_t two = w & 1 ? decode2<TYPE, true>(code, vsc) : decode2<TYPE, false>(code, vsc);
          uint4 &d = vx[(w >> 2) & 1];
          ((w & 3) == 0 ? d.x : (w & 3) == 1 ? d.y : (w & 3) == 2 ? d.z : d.w) = two;
          if ((w & 7) == 7) put_v(cur ^ 1, w >> 3, vx[0], vx[1]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (t + 2 < t_full) {
        fetch_v(t + 2);
        vsc = uniform_load(vsh, ((t + 2) * KT) >> p.shift);
      }
      if (j0 <= see1) absorb_tile<1>(sacc, j0 + KT - 1 > see0, see - j0 - 4 * gg, Vs[cur], vbase, p.c, m_run, lacc, oacc);
    }
  }

  // An infinite key (e5m2 has them) times the two codes of a query's element is inf * 0 or inf - inf where the score is -inf and
  // its key weighs nothing.  Like any NaN that stays in the row's sum, so where there is one the workgroup starts anew, with
  // whole queries for all its tiles (seldom; looking for infinities in the loop would cost every call).
  if (TYPE == SA_CACHE_E5M2 && t_begin < t_full) {
    const float l = lacc[0][0] + lacc[1][0];
    if (__syncthreads_or(l != l)) {
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
      m_run = -INFINITY;
      lacc[0] = lacc[1] = f32x4{};
      whole_tiles(t_begin);
    }
  }

  // ---- non-finite values of V in tiles that only some rows see
  if (t_end > t_masked) {
    __syncthreads();
    for (int t = max(t_begin, t_masked); t < t_end; ++t)
      for (uint64_t bad = __ballot(rowbad[(t - t_masked) * KT + lane] != 0); bad != 0ull; bad &= bad - 1ull)
        add_nonfinite<TYPE>(p, kvh, t * KT + __ffsll((unsigned long long)bad) - 1, head, tok, see, gg, m_run, oacc);
  }
  const float l_run = sum_pair(lacc[0][0] + lacc[1][0]);  // the keys of both lanes of a row
  if (r0 + 32 * wave + q < p.rows) put_row(p, kvh, row, head, tok, sp, gg, m_run, l_run, oacc);
}

// Rows x splits that the scratch holds: two workgroups of 128 rows a compute unit.
size_t max_slots(const Shape &sh) { return (size_t)sh.n_cu * 2 * kRowsMany; }

// Which kernel, and into how many splits the keys go: what orders them is a sum of terms that were each measured with
// 32 heads over 300 to 130 thousand keys and 1 to 2000 tokens (us).  It has no term for the rate of memory or the power limit, so
// for the longest calls it is less than the time (32 for one token of 32 heads at 128K keys, which takes 53).
//                                            few rows      many rows
//   start and end                            5             7
//   keys of a tile (few: of all four waves)  128           64
//   a tile, up to a workgroup a compute unit 0.75          1.15
//   a tile, two, which share it              1.3           1.25
//   start of the second one                  1             1
//   more than two: their number times start and tiles, of which the rows see less than the longest one
//   a join: its launch 3.4, and 1 KB written and read for each row and split at 4.3 TB/s
// The least of them over no splits, as many as give one or two workgroups a compute unit, and in either range where the
// join weighs as much as the tiles that it saves.  Over 169 drawn shapes of 8 to 64 heads the choice is 1.6 % slower than the best of
// both kernels and all splits in the mean, 27 % at worst (9 tokens of 16 heads at 110648 keys, 40.5 us: half the splits 31.9); fixed
// limits on the keys read and the keys a split had been 11.7 us instead of 8.8 (130 tokens at 260 keys), 37.7 instead of 27.6
// (500 tokens of 64 heads at 1000).
struct Plan { bool few; int S; };
Plan plan_of(const Shape &sh, int rows, int tokens, int pos) {
  const float mean = 0.5f + 0.5f * pos / tokens;  // keys that a row sees, against all
  Plan best = {true, 1};
  float least = INFINITY;
  const int64_t all = (int64_t)rows * sh.Hkv;
  for (int few = 1; few >= (rows <= kRowsFew ? 1 : 0); --few) {
    const int per_wg = few ? kRowsFew : kRowsMany, keys = few ? 32 : 64, waves = few ? 4 : 1;  // of a tile; that share out the tiles
    const int64_t wgs = (rows + per_wg - 1) / per_wg * (int64_t)sh.Hkv;
    const int tiles = (tokens + keys - 1) / keys;
    const int top = (int)std::min<int64_t>(std::min(tiles / waves + 1, kMaxSplits), (int64_t)max_slots(sh) / all);
    auto consider = [&](int64_t splits) {
      const int S0 = (int)std::max<int64_t>(1, std::min<int64_t>(splits, top));
      const int share = (tiles + S0 - 1) / S0, S = (tiles + share - 1) / share, per = (share + waves - 1) / waves;
      const float load = (float)wgs * S / sh.n_cu;
      const float start = few ? 5.f : 7.f, two = few ? 1.3f : 1.25f;
      float t = load <= 1.f ? start + per * (few ? 0.75f : 1.15f) : 1.f + std::max(start + per * two, load / 2 * (start + per * two * mean));
      if (S > 1) t += 3.4f + all * S * 0.00023f;
      if (t < least) { least = t; best = {few != 0, S}; }
    };
    consider(1);
    for (int more = 0; more < 2; ++more) {
      const int64_t fill = (more + 1) * (int64_t)sh.n_cu / wgs;
      const float even = std::sqrt((float)tiles / waves * (!few ? 1.2f : more ? 1.3f : 0.75f) / (all * 0.00023f));
      consider(fill);
      consider(std::min<int64_t>(fill, (int64_t)even));
    }
  }
  return best;
}

}  // namespace

void cache_attend_plan(const Shape &sh, int n, int pos, int *rows, int *splits) {
  const Plan plan = plan_of(sh, sh.g * n, pos + n, pos);
  *rows = plan.few ? kRowsFew : kRowsMany;
  *splits = plan.S;
}

size_t attend_scratch_bytes(const Shape &sh) { return max_slots(sh) * (kHeadDim * 4 + 8); }

hipError_t launch_cache_attend(const Shape &sh, const sa_cache &c, sa_rows Q, int n, int pos, sa_rows O,
                               void *scratch, hipStream_t st) {
  AttendArgs a;
  a.Q = (const uint16_t *)Q.data; a.O = (uint16_t *)O.data;
  a.K = (const uint8_t *)c.k; a.V = (const uint8_t *)c.v; a.k_scale = c.k_scale; a.v_scale = c.v_scale;
  a.k_open = (const uint16_t *)c.k_open; a.v_open = (const uint16_t *)c.v_open;
  a.q_hs = Q.head_stride; a.q_rs = Q.row_stride; a.o_hs = O.head_stride; a.o_rs = O.row_stride;
  a.capacity = c.capacity;
  a.g = sh.g; a.Hkv = sh.Hkv; a.rows = sh.g * n;
  a.shift = sh.b == 128 ? 7 : 6;
  a.pos = pos; a.tokens = pos + n; a.closed = a.tokens >> a.shift << a.shift;
  a.c = sh.scale * 1.4426950408889634f;
  const Plan plan = plan_of(sh, a.rows, a.tokens, pos);
  a.tiles = (a.rows + (plan.few ? kRowsFew : kRowsMany) - 1) / (plan.few ? kRowsFew : kRowsMany);
  a.S = plan.S;
  const int64_t wgs = (int64_t)a.tiles * sh.Hkv, all = (int64_t)a.rows * sh.Hkv;
  // Long row tiles first.  Many rows: where every compute unit gets one workgroup and some a second, the second ones in the
  // opposite order, so that the longest share theirs with the shortest (2048 tokens of 32 heads at 0: 49.2 -> 46.1 us, at 5K 178 -> 175).
  // Few rows: the short ones first where a round of one workgroup for most compute units is left at the end, which the long ones
  // have for themselves (700 tokens of 32 heads at 700: 26.3 us, 30.0 the other way; 500 at 0, without such a round, 11.5 and 10.4).
  a.turn = a.tiles;
  if (plan.few) {
    const int64_t left = wgs * a.S % (2 * sh.n_cu);
    a.turn = 2 * left > sh.n_cu && left <= sh.n_cu ? 0 : a.tiles - 1;
  } else if (wgs * a.S > sh.n_cu && wgs * a.S <= 2 * sh.n_cu) {
    a.turn = std::max(1, (int)(sh.n_cu / (sh.Hkv * a.S)));
  }
  a.ml = (float2 *)scratch;
  a.part = (float *)((char *)scratch + max_slots(sh) * 8);
  const unsigned grid = (unsigned)(wgs * a.S);
  const bool e4m3 = c.type == SA_CACHE_E4M3;
  // Probabilities in two parts where a key is read for one or two sets of 32 rows, steps and drafted tokens, which wait for memory or
  // for the launch (32 heads: one token at 128K keys 53.7 us instead of 53.4, at 10K 10.9 and 10.6, at 500 8.3 and 7.7, 16 tokens at 16K 16.3
  // and 15.5).  Chunks of a prompt, bound by the products, take them in bf16 as the sparse prefill does: with two parts 250 tokens at
  // 2200 keys take 21.8 us instead of 18.8, 2048 at 64K in the other kernel 2516 instead of 1652.
  if (plan.few && a.rows <= 2 * kRowsFew) {
    if (e4m3) attend_few_kernel<SA_CACHE_E4M3, 2><<<grid, kThreads, 0, st>>>(a);
    else attend_few_kernel<SA_CACHE_E5M2, 2><<<grid, kThreads, 0, st>>>(a);
  } else if (plan.few) {
    if (e4m3) attend_few_kernel<SA_CACHE_E4M3, 1><<<grid, kThreads, 0, st>>>(a);
    else attend_few_kernel<SA_CACHE_E5M2, 1><<<grid, kThreads, 0, st>>>(a);
  } else {
    if (e4m3) attend_rows_kernel<SA_CACHE_E4M3><<<grid, kThreads, 0, st>>>(a);
    else attend_rows_kernel<SA_CACHE_E5M2><<<grid, kThreads, 0, st>>>(a);
  }
  launch_join(a, all, st);
  return hipGetLastError();
}

}  // namespace sa
