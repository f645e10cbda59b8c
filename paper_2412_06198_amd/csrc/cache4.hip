// The key/value cache in 4 bits: appending tokens; and reading either cache back into bf16 tensors.
//
// A row (one token of a KV head) has four groups of 32 adjacent elements, each with codes x / s in e2m1 (magnitudes 0 .5 1 1.5 2 3 4 6)
// and one scale s = 2^e as a byte: the operands that the scaled matrix instructions take.  A group is the smallest that they know, since with one
// bit of mantissa it is the scale that has to follow the values; a row's own scales make a token independent of its neighbours, so there
// is no open block and a token may be written again.  x / s and code * s are exact, the rounding to the code is the only one.
// Both directions read and write everything once: the bound is HBM.  A row is taken by 16 lanes, 8 elements each, so that every access of
// a wave is contiguous (16 bytes a lane in bf16, 4 in codes); a group is four lanes, whose largest magnitude is two lane moves.  128K tokens of 8 heads, 680 MB: 110 us
// to append, 109 to read back (6.2 TB/s; a device copy moves 5.1), 128 to read back from 8 bits (6.3 TB/s).  What is read back goes past the caches
// (120 us with ordinary stores), the codes do not, since they are read next (10K tokens stored and read back 18.8 to 19.6 us, 21.0 past them).
#include "cache4_codes.h"
#include "cache_codes.h"
#include "sa_internal.h"

namespace sa {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = kThreads / 16;  // rows that a workgroup takes at a time
constexpr int U = 2;                  // times, all reads of which are on their way at once (4: 128K tokens appended in 116 us instead of 110, read back in 120, 109; 1: 114, 123)

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Append4Args {
  const uint16_t *src[2];  // K, V
  int64_t hs[2], rs[2];
  uint8_t *codes[2];
  uint32_t *scale[2];      // a row's four bytes
  int64_t n, pos, capacity;
};

template <int CTRL>
__device__ inline uint32_t row_moved(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false); }

// Grid (ceil(n / 32), KV heads, K or V).
__global__ __launch_bounds__(kThreads) void append4_kernel(Append4Args p) {
  const int side = blockIdx.z, h = blockIdx.y, ln = threadIdx.x & 15;
  const int64_t t0 = (int64_t)blockIdx.x * (kRows * U) + (threadIdx.x >> 4);
  const uint16_t *src = p.src[side] + h * p.hs[side] + ln * 8;
  uint4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = *(const uint4 *)(src + min(t0 + kRows * u, p.n - 1) * p.rs[side]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t t = t0 + kRows * u;
    if (t >= p.n) return;
    uint32_t m = max_halves(max_halves(x[u].x & 0x7FFF7FFFu, x[u].y & 0x7FFF7FFFu), max_halves(x[u].z & 0x7FFF7FFFu, x[u].w & 0x7FFF7FFFu));
    m = max_halves(m, row_moved<0xB1>(m));  // the lane beside
    m = max_halves(m, row_moved<0x4E>(m));  // and the other two of the group
    m = max(m & 0xFFFFu, m >> 16);
    const bool number = m < 0x7F80u;
    const uint32_t byte = number ? (uint32_t)(scale_exponent4(m) + 127) : kNanScale;
    const uint32_t codes = number ? encode4_8(x[u], scale4(byte)) : 0u;
    uint32_t word = byte << (8 * (ln >> 2));
    word |= row_moved<0x124>(word);  // of the lanes 4 and 8 further round the row
    word |= row_moved<0x128>(word);
    const int64_t row = h * p.capacity + p.pos + t;
    *(uint32_t *)(p.codes[side] + row * kRow4 + ln * 4) = codes;
    if (ln == 0) p.scale[side][row] = word;
  }
}

struct ReadArgs {
  const uint8_t *codes[2];
  const void *scale[2];
  const uint16_t *open[2];
  uint16_t *dst[2];
  int64_t hs[2], rs[2];
  int64_t n, pos, capacity, closed;  // closed: tokens in full blocks
  int shift;                         // log2 of the block
};

constexpr int kType4 = -1;  // beside the types of the 8-bit cache

// Grid as above, over the sides that are wanted.
template <int TYPE>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs p) {
  const int side = blockIdx.z, h = blockIdx.y, ln = threadIdx.x & 15;
  const int64_t t0 = (int64_t)blockIdx.x * (kRows * U) + (threadIdx.x >> 4);
  uint16_t *dst = p.dst[side] + h * p.hs[side] + ln * 8;
  u32x4 y[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t t = p.pos + min(t0 + kRows * u, p.n - 1), row = h * p.capacity + t;
    if constexpr (TYPE == kType4) {
      y[u][0] = *(const uint32_t *)(p.codes[side] + row * kRow4 + ln * 4);
      y[u][1] = ((const uint32_t *)p.scale[side])[row];
    } else if (t < p.closed) {
      const uint2 c = *(const uint2 *)(p.codes[side] + row * kHeadDim + ln * 8);
      y[u][0] = c.x;
      y[u][1] = c.y;
      y[u][2] = __float_as_uint(((const float *)p.scale[side])[h * (p.capacity >> p.shift) + (t >> p.shift)]);
    } else {
      y[u] = *(const u32x4 *)(p.open[side] + (((int64_t)h << p.shift) + (t - p.closed)) * kHeadDim + ln * 8);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t t = t0 + kRows * u;
    if (t >= p.n) return;
    if constexpr (TYPE == kType4) {
      const uint4 r = decode4_8(y[u][0], scale4(y[u][1] >> (8 * (ln >> 2)) & 0xFFu));
      y[u] = u32x4{r.x, r.y, r.z, r.w};
    } else if (p.pos + t < p.closed) {
      const float s = __uint_as_float(y[u][2]);
      y[u] = u32x4{decode2<TYPE, false>(y[u][0], s), decode2<TYPE, true>(y[u][0], s), decode2<TYPE, false>(y[u][1], s), decode2<TYPE, true>(y[u][1], s)};
    }
    __builtin_nontemporal_store(y[u], (u32x4 *)(dst + t * p.rs[side]));
  }
}

template <int TYPE>
hipError_t launch_read(ReadArgs &a, const void *const (&codes)[2], const void *const (&scale)[2], const void *const (&open)[2], const sa_rows (&to)[2],
                       int heads, hipStream_t st) {
  int sides = 0;
  for (int i = 0; i < 2; ++i) {
    if (!to[i].data) continue;
    a.codes[sides] = (const uint8_t *)codes[i]; a.scale[sides] = scale[i]; a.open[sides] = (const uint16_t *)open[i];
    a.dst[sides] = (uint16_t *)to[i].data; a.hs[sides] = to[i].head_stride; a.rs[sides] = to[i].row_stride;
    ++sides;
  }
  read_kernel<TYPE><<<dim3((unsigned)((a.n + kRows * U - 1) / (kRows * U)), (unsigned)heads, (unsigned)sides), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache4_append(const Shape &sh, const sa_cache4 &c, sa_rows K, sa_rows V, int64_t n, int64_t pos, hipStream_t st) {
  Append4Args a;
  a.src[0] = (const uint16_t *)K.data; a.src[1] = (const uint16_t *)V.data;
  a.hs[0] = K.head_stride; a.hs[1] = V.head_stride; a.rs[0] = K.row_stride; a.rs[1] = V.row_stride;
  a.codes[0] = (uint8_t *)c.k; a.codes[1] = (uint8_t *)c.v;
  a.scale[0] = (uint32_t *)c.k_scale; a.scale[1] = (uint32_t *)c.v_scale;
  a.n = n; a.pos = pos; a.capacity = c.capacity;
  append4_kernel<<<dim3((unsigned)((n + kRows * U - 1) / (kRows * U)), (unsigned)sh.Hkv, 2), kThreads, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache4_read(const Shape &sh, const sa_cache4 &c, sa_rows K, sa_rows V, int64_t n, int64_t pos, hipStream_t st) {
  ReadArgs a = {};
  a.n = n; a.pos = pos; a.capacity = c.capacity;
  return launch_read<kType4>(a, {c.k, c.v}, {c.k_scale, c.v_scale}, {nullptr, nullptr}, {K, V}, sh.Hkv, st);
}

hipError_t launch_cache_read(const Shape &sh, const sa_cache &c, int64_t tokens, sa_rows K, sa_rows V, int64_t n, int64_t pos, hipStream_t st) {
  ReadArgs a = {};
  a.n = n; a.pos = pos; a.capacity = c.capacity;
  a.shift = sh.b == 128 ? 7 : 6;
  a.closed = tokens >> a.shift << a.shift;
  if (c.type == SA_CACHE_E4M3) return launch_read<SA_CACHE_E4M3>(a, {c.k, c.v}, {c.k_scale, c.v_scale}, {c.k_open, c.v_open}, {K, V}, sh.Hkv, st);
  return launch_read<SA_CACHE_E5M2>(a, {c.k, c.v}, {c.k_scale, c.v_scale}, {c.k_open, c.v_open}, {K, V}, sh.Hkv, st);
}

}  // namespace sa
