// The key/value cache in 8 bits: appending tokens.
//
// A block of b tokens that is full has, for each KV head, codes x / s in 8-bit floating point and one scale s, the
// least power of two with max|x| <= s * (largest of the type).  A power of two costs a floating-point type no
// precision, only range, and makes every step exact but the one rounding to the code: x / s and code * s are exact,
// a key out of the cache is a bf16 value, and a reader may multiply by s wherever it suits it.  The open block
// stays bf16 until it is full, so that a token is rounded once, by a scale that fits its whole block, however many
// calls bring the block.
// Every value is read once and written once: the bound is HBM (128K tokens of 8 heads, 805 MB, 138 us: 5.8 TB/s; a device copy
// moves 5.1).  A workgroup holds a block of one head in registers
// (16 or 32 KB), takes the largest magnitude and writes codes, so nothing is read twice.
#include "cache_codes.h"
#include "sa_internal.h"

namespace sa {
namespace {

constexpr int kThreads = 256;
constexpr int kPieceRows = kThreads / 8;  // rows that a workgroup holds in one piece a thread: 16 elements each

struct AppendArgs {
  const uint16_t *src[2];  // K, V
  int64_t hs[2], rs[2];
  uint8_t *codes[2];
  float *scale[2];
  uint16_t *open[2];
  int64_t pos, end;        // tokens before, tokens after
  int64_t capacity;
  int shift;               // log2 of the block
};

struct Piece { uint4 x[2]; };
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline uint32_t max_halves(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Magnitudes of two bf16 values; FINITE: those of infinities and NaN count 0.
template <bool FINITE>
__device__ inline uint32_t magnitudes(uint32_t w) {
  const uint32_t t = w & 0x7FFF7FFFu;
  if (!FINITE) return t;
  const uint32_t bad = (t + 0x00800080u) & 0x80008000u;  // exponent 255
  return t & ~((bad << 1) - (bad >> 15));                // 0xFFFF where bad
}
template <bool FINITE>
__device__ inline uint32_t largest(const Piece &p) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    m = max_halves(m, magnitudes<FINITE>(p.x[i].x));
    m = max_halves(m, magnitudes<FINITE>(p.x[i].y));
    m = max_halves(m, magnitudes<FINITE>(p.x[i].z));
    m = max_halves(m, magnitudes<FINITE>(p.x[i].w));
  }
  return m;
}
// The larger half, over the workgroup, on every thread.
__device__ inline uint32_t over_workgroup(uint32_t m, uint32_t *wave_max) {
  m = max(m & 0xFFFFu, m >> 16);
  for (int e = 32; e >= 1; e >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, e));
  if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3]));
  __syncthreads();
  return m;
}

// Grid (blocks that the tokens touch, KV heads, K or V), 256 threads.
template <int TYPE, int PIECES>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs p) {
  __shared__ uint32_t wave_max[4];
  const int side = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int b = 1 << p.shift;
  const int64_t first = p.pos >> p.shift, block = first + blockIdx.x, last = p.end >> p.shift;
  const uint16_t *src = p.src[side] + h * p.hs[side];
  uint16_t *open = p.open[side] + (int64_t)h * b * kHeadDim;
  const int row = tid >> 3, el = (tid & 7) * 16;
  // tokens lo .. hi - 1 of `block` from the source into the open block
  auto copy = [&](int64_t of, int64_t lo, int64_t hi) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int r = kPieceRows * i + row;
      const int64_t t = (of << p.shift) + r;
      if (t >= lo && t < hi) {
        const uint4 *x = (const uint4 *)(src + (t - p.pos) * p.rs[side] + el);
        uint4 *y = (uint4 *)(open + r * kHeadDim + el);
        y[0] = x[0];
        y[1] = x[1];
      }
    }
  };
  // The last, open block is written by its own workgroup, unless the first block's reads what was open before
  // the call: then that one writes it too, when it has read.
  const bool in_turn = (p.pos & (b - 1)) != 0 && last > first;
  if (block == last) {
    if (!in_turn) copy(block, p.pos, p.end);
    return;
  }
  Piece x[PIECES];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int r = kPieceRows * i + row;
    const int64_t t = (block << p.shift) + r;
    const uint4 *at = (const uint4 *)(t < p.pos ? open + r * kHeadDim + el : src + (t - p.pos) * p.rs[side] + el);
    x[i].x[0] = at[0];
    x[i].x[1] = at[1];
  }
#pragma unroll
  for (int i = 0; i < PIECES; ++i) m = max_halves(m, largest<false>(x[i]));
  m = over_workgroup(m, wave_max);
  if (m >= 0x7F80u) {  // infinities or NaN: the others alone make the scale
    m = 0;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) m = max_halves(m, largest<true>(x[i]));
    m = over_workgroup(m, wave_max);
  }
  const int e = scale_exponent<TYPE>(m);
  const float inverse = __uint_as_float((uint32_t)(127 - e) << 23);
  uint8_t *codes = p.codes[side] + ((int64_t)h * p.capacity + (block << p.shift)) * kHeadDim;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    u32x4 y;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      y[2 * k] = encode4<TYPE>(x[i].x[k].x, x[i].x[k].y, inverse);
      y[2 * k + 1] = encode4<TYPE>(x[i].x[k].z, x[i].x[k].w, inverse);
    }
    __builtin_nontemporal_store(y, (u32x4 *)(codes + (kPieceRows * i + row) * kHeadDim + el));  // 144 -> 138 us at 128K tokens
  }
  if (tid == 0) p.scale[side][h * (p.capacity >> p.shift) + block] = __uint_as_float((uint32_t)(127 + e) << 23);
  if (block == first && in_turn) copy(last, last << p.shift, p.end);
}

template <int TYPE>
void launch(const AppendArgs &a, dim3 grid, hipStream_t st) {
  if (a.shift == 7) append_kernel<TYPE, 128 / kPieceRows><<<grid, kThreads, 0, st>>>(a);
  else append_kernel<TYPE, 64 / kPieceRows><<<grid, kThreads, 0, st>>>(a);
}

}  // namespace

hipError_t launch_cache_append(const Shape &sh, const sa_cache &c, sa_rows K, sa_rows V, int64_t n, int64_t pos,
                               hipStream_t st) {
  AppendArgs a;
  a.src[0] = (const uint16_t *)K.data; a.src[1] = (const uint16_t *)V.data;
  a.hs[0] = K.head_stride; a.hs[1] = V.head_stride; a.rs[0] = K.row_stride; a.rs[1] = V.row_stride;
  a.codes[0] = (uint8_t *)c.k; a.codes[1] = (uint8_t *)c.v;
  a.scale[0] = c.k_scale; a.scale[1] = c.v_scale;
  a.open[0] = (uint16_t *)c.k_open; a.open[1] = (uint16_t *)c.v_open;
  a.pos = pos; a.end = pos + n; a.capacity = c.capacity;
  a.shift = sh.b == 128 ? 7 : 6;
  const dim3 grid((unsigned)(((a.end - 1) >> a.shift) - (pos >> a.shift) + 1), (unsigned)sh.Hkv, 2);
  if (c.type == SA_CACHE_E4M3) launch<SA_CACHE_E4M3>(a, grid, st);
  else launch<SA_CACHE_E5M2>(a, grid, st);
  return hipGetLastError();
}

}  // namespace sa
