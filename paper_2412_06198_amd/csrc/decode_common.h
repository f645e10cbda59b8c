// What the two decode steps (K and V in bf16, and in the 8-bit cache) share: sums over the lanes, partial results of
// a head, the count of the workgroups that have written theirs, and their merge.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sa {

constexpr int kPartStride = 132;  // floats per partial: max, sum, 2 (first one: arrival counter, others: 0), 128 outputs

// A head's arrival counter lives in floats 2 and 3 of its first partial: the step's token in the upper 48
// bits, in the lower 16 the number of workgroups that have arrived.  The memory may hold anything: what the
// caller's workspace was used for before, or the count of a step that overlapped another one or never ended.
// A step takes only its own token for a count: a head's first workgroup puts the token there while its rows are
// on their way, one that arrives before that does it itself, and nothing is read from what was left.  Each
// launch has a token of its own, so that no clearing launch is needed; a recorded one repeats its token with
// every replay, so there the counters are cleared by a launch before it (8 heads, 4096 tokens: 8.4 us a
// recorded step instead of 6.6; a count that the last one to arrive put back to 0 cost 0.1 us less, and what an
// overlapping step left there stayed for good).
constexpr int kCountBits = 16;

// A reduction over the four 16-lane slots of a wave, on each lane.
template <typename F>
__device__ inline float over_slots(float x, F f) {
  const unsigned a = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const unsigned r0 = r[0], r1 = r[1];
  const unsigned c = __float_as_uint(f(__uint_as_float(r0), __uint_as_float(r1)));
  const auto s = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  const unsigned s0 = s[0], s1 = s[1];
  return f(__uint_as_float(s0), __uint_as_float(s1));
}

__device__ inline void unpack8(const uint4 x, float (&f)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(w[e] << 16);
    f[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}

// The value of another lane of the same 16.
template <int CTRL>
__device__ inline float row_move(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}

// Partial results cross workgroups inside the launch by agent-scope accesses, which pass the L2 caches
// by: nothing has to be written back or invalidated on the way (fences at that scope cost 40 us here).  They
// are ordered before the arrival by vmcnt(0) and the workgroup's barrier, see the top of index.hip.
__device__ inline void put(float *p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline float get(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Merge n <= 64 partials of a head, normalise, round to bf16: 256 threads, thread (k0, d) takes the outputs d
// of partials k0, k0 + 2, ...  All reads are on their way before the first is needed.  A sum that is not positive (NaN
// among the scores) gives 0, or with KEEP_NAN what the division does.
template <bool KEEP_NAN>
__device__ inline void merge(const float *src, int n, float *wgt, float *s_L, float *half, uint16_t *o) {
  const int tid = threadIdx.x, d = tid & 127, k0 = tid >> 7;
  float mk = -INFINITY, lk = 0.f;
  if (tid < n) {
    mk = get(src + (size_t)tid * kPartStride);
    lk = get(src + (size_t)tid * kPartStride + 1);
  }
  float x[32];
  // Places past the end weigh 0 and read the 0 that the last partial holds for them: anything else could be
  // infinite.  (Masks on x after the reads cost 0.3 us.)
  const int none = (n - 1) * kPartStride + 2;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if (8 * (i / 8) * 2 < n) x[i] = get(src + (k0 + 2 * i < n ? (k0 + 2 * i) * kPartStride + 4 + d : none));  // by eights
    else x[i] = 0.f;
  }
  if (tid < 64) {
    float M = mk;
    for (int e = 32; e >= 1; e >>= 1) M = fmaxf(M, __shfl_xor(M, e));
    const float w = mk == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mk - M);
    float L = lk * w;
    for (int e = 32; e >= 1; e >>= 1) L += __shfl_xor(L, e);
    wgt[tid] = w;  // 0 from n on
    if (tid == 0) *s_L = L;
  }
  __syncthreads();
  float O = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i)
    O = __builtin_fmaf(x[i], wgt[k0 + 2 * i], O);
  if (k0) half[d] = O;
  __syncthreads();
  if (k0) return;
  O += half[d];
  const float L = *s_L;
  const __bf16 r = (__bf16)(KEEP_NAN || L > 0.f ? O / L : 0.f);
  o[d] = __builtin_bit_cast(uint16_t, r);
}

// What one lane has written to LDS before is read by the others of its wave after it, and the other way round.
__device__ inline void wave_lds_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The token into a head's counter, which held `seen`, unless a workgroup of this step has been there.
__device__ inline void claim(uint64_t *arrived, uint64_t seen, uint64_t token) {
  if ((seen ^ token) >> kCountBits)
    (void)__hip_atomic_compare_exchange_strong(arrived, &seen, token, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
}

// Counts the calling workgroup; whether it is the last of the head's n.
__device__ inline bool arrive(uint64_t *arrived, uint64_t token, int n) {
  uint64_t before = __hip_atomic_fetch_add(arrived, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  while ((before ^ token) >> kCountBits) {  // added to a value that is not this step's: nobody has been here yet
    uint64_t cur = before + 1;                // ends: an exchange only fails where a workgroup has changed the counter
    if (__hip_atomic_compare_exchange_strong(arrived, &cur, token + 1, __ATOMIC_RELAXED, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT))
      before = token;  // this one put the token there, and itself
    else if ((cur ^ token) >> kCountBits)
      before = cur - 1;
    else
      before = __hip_atomic_fetch_add(arrived, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  return before == token + (uint64_t)(n - 1);
}

// The arrival counters of all heads, before a recorded step.
static __global__ void clear_arrivals_kernel(float *part, int Hq, int S) {
  if ((int)threadIdx.x < Hq) *(uint64_t *)(part + (size_t)threadIdx.x * S * kPartStride + 2) = 0;
}

}  // namespace sa
