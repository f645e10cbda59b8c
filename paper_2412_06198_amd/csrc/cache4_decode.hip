// One decode step over the prefill index, K and V out of the 4-bit cache: the keys, their order and the launch are those of the step
// over the 8-bit cache (cache_decode.hip), half the bytes.  A key is read by 16 lanes as 64 bytes of codes of K and of V, and the two bytes of
// their group's scales, which the conversion to fp32 applies.  There is no open block, so all keys are rows of one kind.  The bound is a launch and the
// round trips to memory that follow one another, as there: 8 heads at 4K tokens 6.6 to 6.9 us with the host's call, 32 heads at 128K tokens, 3 %
// kept, 11.0 to 11.1.
#include <algorithm>

#include "cache4_codes.h"
#include "decode_common.h"
#include "sa_internal.h"

namespace sa {
namespace {

struct Cache4DecArgs {
  const uint16_t *q;
  const uint8_t *K, *V;
  const uint8_t *k_scale, *v_scale;
  uint16_t *o;
  const int32_t *n_cols, *cols, *n_offs, *offs, *rowptr, *blkcols;
  float *part;
  int Hq, g, N, nb, shift, k_v, k_s, cap_b, S, pos;
  int64_t capacity;
  float c;  // softmax scale * log2(e)
  uint64_t token;
};

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kLanes = 16, kSlots = 64 / kLanes;  // lanes of a key, keys that a wave reads at once
// Rows of K and of V that a lane has in flight per step.  8: 0.1 to 0.7 us slower from 4K tokens on, 2: up to 0.9.  8 lanes a key, 8 bytes
// each: 0.2 us faster at 32 heads and 128K tokens, 0.1 to 0.6 slower elsewhere.
constexpr int U = 4;
constexpr int kStep = kSlots * U;
constexpr int kRing = 128;                        // keys of a wave that are resolved and not yet read: 15 + 64 at most
constexpr int kMinChunk = kWaves * kStep;         // keys of a workgroup: one step of each wave

// Sum over 16 lanes, on each of them: partners at distance 8, 7, 2 and 1.
__device__ inline float sum16(float x) {
  x += row_move<0x128>(x);
  x += row_move<0x141>(x);
  x += row_move<0x4E>(x);
  x += row_move<0xB1>(x);
  return x;
}

// A head's key list, in this order: keys of the kept blocks, columns, diagonal keys, generated keys; and how it is shared out:
// workgroups 0 .. n - 1 take `chunk` keys each.
struct KeyList {
  int e0, nblk, nc, no, n0, n1, n2, total, chunk, n;
};
__device__ inline KeyList key_list(const Cache4DecArgs &p, int h) {
  KeyList k;
  const int32_t *rp = p.rowptr + (size_t)h * (p.nb + 1);
  k.e0 = min(max(rp[p.nb - 1], 0), p.cap_b);
  k.nblk = min(max(rp[p.nb], k.e0), p.cap_b) - k.e0;
  k.nc = min(max(p.n_cols[h], 0), p.k_v);
  k.no = min(max(p.n_offs[h], 0), p.k_s);
  k.n0 = k.nblk << p.shift;
  k.n1 = k.n0 + k.nc;
  k.n2 = k.n1 + k.no;
  k.total = k.n2 + p.pos + 1 - p.N;
  k.chunk = max(((k.total + p.S - 1) / p.S + 15) / 16 * 16, kMinChunk);
  k.n = (k.total + k.chunk - 1) / k.chunk;  // <= S, and at least 1: the query's own key is in the list
  return k;
}

// grid (S, Hq), 256 threads.  Each wave walks a quarter of the workgroup's keys by itself: 64 lanes resolve 64
// list places (which key, does it count here), the keys that count queue up in the wave's ring, and a step
// reads the rows of 16 of them, slot s of 16 lanes every fourth one, lane ln elements 8 ln .. 8 ln + 7.
__global__ __launch_bounds__(kThreads) void cache4_decode_kernel(Cache4DecArgs p) {
  __shared__ __attribute__((aligned(16))) uint32_t blkbm[kMaxSeq / 64 / 32];  // key blocks kept for the last row block
  __shared__ __attribute__((aligned(16))) uint32_t colbm[kMaxSeq / 32];       // selected key columns
  __shared__ int ring[kWaves][kRing];                                         // keys
  __shared__ float sm[kWaves], sl[kWaves];
  __shared__ __attribute__((aligned(16))) float so[kWaves][kHeadDim];
  __shared__ float wgt[64], s_L;
  __shared__ unsigned s_last;
  const int sp = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, kvh = h / p.g;
  const int N = p.N, nb = p.nb, b = 1 << p.shift, shift = p.shift;
  const int lane = tid & 63, ln = tid & (kLanes - 1), slot = lane / kLanes, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint4 qx = *(const uint4 *)(p.q + (size_t)h * kHeadDim + ln * 8);
  const KeyList L = key_list(p, h);
  if (sp >= L.n) return;
  float *part = p.part + (size_t)h * gridDim.x * kPartStride;
  uint64_t *arrived = (uint64_t *)(part + 2);
  const bool counts = tid == kThreads - 1, claims = counts && sp == 0;  // the thread that counts the arrival
  uint64_t seen = 0;
  if (claims) seen = __hip_atomic_load(arrived, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

  float qv[8], m = -INFINITY, l = 0.f, acc[8];
  unpack8(qx, qv);
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.f;
  // The softmax step of U keys a slot, of which the first n of the wave's count: key(u, f) and val(u, f) give this lane's
  // elements of a row.
  auto absorb = [&](auto key, auto val, int n) {
    float s[U], m_new = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float kf[8], dot = 0.f;
      key(u, kf);
#pragma unroll
      for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(kf[e], qv[e], dot);
      s[u] = kSlots * u + slot < n ? sum16(dot) * p.c : -INFINITY;
      m_new = fmaxf(m_new, s[u]);
    }
    const float m_ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m - m_ref);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float pv = __builtin_amdgcn_exp2f(s[u] - m_ref);
      float vf[8];
      val(u, vf);
      l += pv;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = __builtin_fmaf(pv, vf[e], acc[e]);
    }
  };

  {
    const int32_t *bc = p.blkcols + (size_t)h * p.cap_b + L.e0;
    const int32_t *colp = p.cols + (size_t)h * p.k_v;
    const int32_t *offp = p.offs + (size_t)h * p.k_s;
    const int t_begin = sp * L.chunk, t_end = min(t_begin + L.chunk, L.total);
    const int share = ((t_end - t_begin + kWaves - 1) / kWaves + kStep - 1) / kStep * kStep;
    int t_next = min(t_begin + wave * share, t_end);
    const int t_stop = min(t_next + share, t_end);
    auto entry = [&](int t) {  // what the list says at a place; generated keys stand in no list
      const int32_t *src = t < L.n0 ? bc + (t >> shift) : t < L.n1 ? colp + (t - L.n0) : offp + (t - L.n1);
      return t < t_stop && t < L.n2 ? *src : -1;
    };
    int ent = entry(t_next + lane);
    // A key counts where it first appears in the list: columns and diagonal keys are screened by the kept
    // blocks, diagonal keys by the columns too.  Only workgroups with such keys build the bitmaps.
    const bool need_blk = t_begin < L.n2 && t_end > L.n0, need_cols = t_begin < L.n2 && t_end > L.n1 && L.nc > 0 && L.no > 0;
    if (need_blk) {
      for (int i = tid; i < (nb + 127) / 128; i += kThreads) ((uint4 *)blkbm)[i] = make_uint4(0u, 0u, 0u, 0u);
      if (need_cols)
        for (int i = tid; i < (N + 127) / 128; i += kThreads) ((uint4 *)colbm)[i] = make_uint4(0u, 0u, 0u, 0u);
      __syncthreads();
      for (int e = tid; e < L.nblk; e += kThreads) {
        const int C = bc[e];
        if (C >= 0 && C < nb) atomicOr(&blkbm[C >> 5], 1u << (C & 31));
      }
      if (need_cols)
        for (int i = tid; i < L.nc; i += kThreads) {
          const int c = colp[i];
          if (c >= 0 && c < N) atomicOr(&colbm[c >> 5], 1u << (c & 31));
        }
      __syncthreads();
    }
    auto kept_block = [&](int key) { const int C = key >> shift; return ((blkbm[C >> 5] >> (C & 31)) & 1u) != 0u; };
    const uint8_t *Kh = p.K + (size_t)kvh * p.capacity * kRow4 + ln * 4;
    const uint8_t *Vh = p.V + (size_t)kvh * p.capacity * kRow4 + ln * 4;
    const uint8_t *ksh = p.k_scale + (size_t)kvh * p.capacity * kScales4 + (ln >> 2), *vsh = p.v_scale + (size_t)kvh * p.capacity * kScales4 + (ln >> 2);
    int put_at = 0, get_at = 0;  // of the ring, uniform
    auto resolve = [&] {         // until a step is full or the list at its end
      while (put_at - get_at < kStep && t_next < t_stop) {
        const int t = t_next + lane;
        int j = -1;
        if (t < L.n0) {
          if (ent >= 0 && ent < nb) j = (ent << shift) + (t & (b - 1));
        } else if (t < L.n1) {
          if (ent >= 0 && ent < N && !kept_block(ent)) j = ent;
        } else if (t < L.n2) {
          const int jj = p.pos - ent;
          if (ent >= 0 && jj >= 0 && jj < N && !kept_block(jj) && !(need_cols && ((colbm[jj >> 5] >> (jj & 31)) & 1u)))
            j = jj;
        } else if (t < t_stop) {
          j = N + (t - L.n2);
        }
        t_next += 64;
        ent = entry(t_next + lane);
        const uint64_t live = __ballot(j >= 0);
        const int at = put_at + __builtin_amdgcn_mbcnt_hi((uint32_t)(live >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)live, 0u));
        if (j >= 0) ring[wave][at & (kRing - 1)] = j;
        put_at += __popcll(live);
      }
      return put_at > get_at;
    };
    struct Rows { uint32_t k[U], v[U]; uint8_t sk[U], sv[U]; int n; };
    auto fetch = [&](Rows &r) {
      r.n = min(put_at - get_at, kStep);
      wave_lds_sync();
#pragma unroll
      for (int u = 0; u < U; ++u) {  // a place without a key reads the last key again
        const int j = ring[wave][(get_at + min(kSlots * u + slot, r.n - 1)) & (kRing - 1)];
        r.k[u] = *(const uint32_t *)(Kh + (size_t)j * kRow4);
        r.v[u] = *(const uint32_t *)(Vh + (size_t)j * kRow4);
        r.sk[u] = ksh[(size_t)j * kScales4];
        r.sv[u] = vsh[(size_t)j * kScales4];
      }
      wave_lds_sync();
      get_at += r.n;
    };
    auto attend = [&](Rows &r) {
      if (r.n < kStep) {  // the last step: a place without a key weighs 0, and 0 x NaN is not 0
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (kSlots * u + slot >= r.n) r.sv[u] = 127;
      }
      absorb([&](int u, float (&f)[8]) { decode4_8f(r.k[u], scale4(r.sk[u]), f); }, [&](int u, float (&f)[8]) { decode4_8f(r.v[u], scale4(r.sv[u]), f); }, r.n);
    };
    // the rows of a step are read while the step before is computed
    Rows even, odd;
    if (resolve()) {
      fetch(even);
      if (claims) claim(arrived, seen, p.token);
      for (;;) {
        const bool more = resolve();
        if (more) fetch(odd);
        attend(even);
        if (!more) break;
        const bool again = resolve();
        if (again) fetch(even);
        attend(odd);
        if (!again) break;
      }
    }
  }
  // the four slots of a wave, then the waves
  const float Mw = over_slots(m, [](float x, float y) { return fmaxf(x, y); });
  const float ww = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - Mw);
  const auto add = [](float x, float y) { return x + y; };
  l = over_slots(l * ww, add);
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = over_slots(acc[e] * ww, add);
  if (lane < kLanes) {
    if (lane == 0) { sm[wave] = Mw; sl[wave] = l; }
    *(float4 *)&so[wave][ln * 8] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    *(float4 *)&so[wave][ln * 8 + 4] = make_float4(acc[4], acc[5], acc[6], acc[7]);
  }
  __syncthreads();
  if (tid < kHeadDim) {
    float M = -INFINITY;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) M = fmaxf(M, sm[k]);
    float lsum = 0.f, O = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float w = sm[k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[k] - M);  // no key, or none but NaN: sums of 0 or NaN
      lsum += sl[k] * w;
      O += so[k][tid] * w;
    }
    if (L.n == 1) {  // the only workgroup of the head
      const __bf16 r = (__bf16)(O / lsum);
      p.o[(size_t)h * kHeadDim + tid] = __builtin_bit_cast(uint16_t, r);
    } else {
      float *dst = part + (size_t)sp * kPartStride;
      if (tid == 0) { put(dst, M); put(dst + 1, lsum); }
      if (tid == 1 && sp > 0) put(dst + 2, 0.f);  // see merge; dst[2], dst[3] of the first one: the counter
      put(dst + 4 + tid, O);
    }
  }
  if (L.n == 1) return;
  // ---- the last one to arrive merges; nobody waits
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this thread's partials have been performed
  __syncthreads();
  if (counts) s_last = arrive(arrived, p.token, L.n);
  __syncthreads();
  asm volatile("" ::: "memory");
  if (s_last) merge<true>(part, L.n, wgt, &s_L, so[0], p.o + (size_t)h * kHeadDim);
}

// Partials of a head: two workgroups of four waves a compute unit in all.  Three: 32 heads at 16K tokens and a tenth kept 8.9 us instead of 7.8, at
// 4K and a fifth 9.9 instead of 8.6 (at 128K 10.9 instead of 11.1); one and a half: 8.5, 9.6, 12.4.
int splits(const Shape &sh) { return std::max(2, std::min(64, 512 / sh.Hq)); }

}  // namespace

size_t cache4_decode_partial_bytes(const Shape &sh) { return (size_t)sh.Hq * splits(sh) * kPartStride * 4; }

hipError_t launch_cache4_decode(const Shape &sh, float *partials, const sa_cache4 &c, const uint16_t *q, sa_index idx,
                                int pos, uint16_t *o, hipStream_t st) {
  Cache4DecArgs a;
  a.q = q; a.K = (const uint8_t *)c.k; a.V = (const uint8_t *)c.v; a.k_scale = c.k_scale; a.v_scale = c.v_scale; a.o = o;
  a.n_cols = idx.n_cols; a.cols = idx.cols; a.n_offs = idx.n_offs; a.offs = idx.offs;
  a.rowptr = idx.rowptr; a.blkcols = idx.blkcols;
  a.part = partials;
  a.Hq = sh.Hq; a.g = sh.g; a.N = sh.N; a.nb = sh.nb; a.shift = sh.b == 128 ? 7 : 6; a.k_v = sh.k_v; a.k_s = sh.k_s;
  a.cap_b = sh.cap_b; a.pos = pos; a.capacity = c.capacity;
  a.c = sh.scale * 1.4426950408889634f;
  a.token = next_decode_token();
  // Workgroups per head: no more than the partials have room for, or than have a step's keys in the longest list that the budgets allow.
  const int64_t longest = (int64_t)pos + 1 + sh.k_v + sh.k_s;
  a.S = (int)std::min<int64_t>(splits(sh), (longest + kMinChunk - 1) / kMinChunk);
  if (decode_recorded(st)) clear_arrivals_kernel<<<1, kMaxHeads, 0, st>>>(partials, sh.Hq, a.S);
  cache4_decode_kernel<<<dim3(a.S, sh.Hq), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace sa
