// Rotary positions: pair i of a row at position p is turned by the angle p w_i,
//   (x, y) -> (x cos - y sin, x sin + y cos).
// Every element is read and written once and nothing else is: the bound is HBM (128K tokens of 40 heads 446 us, 6.0 TB/s
// moved, where a device copy reaches 5.1; 429 in a replayed loop), and the launch for a single token (2.2 us).  The sines and cosines of a token
// serve all heads of Q and K, so a thread takes W pairs of one token and walks a range of heads with them in registers.
// Angles are kept as fractions of a turn in 64-bit fixed point: position times frequency modulo one turn is then one
// wrapping integer product, to 2^-32 of a turn for any position, where fp32 radians are off by a hundredth at 256K tokens.  As an
// fp32 number, 24 bits of half a turn, it is off by 2^-26 of a turn more at most.
#include <algorithm>
#include <cmath>
#include <new>

#include "sa_internal.h"

struct sa_rotary {
  sa_rotary_config cfg;
  sa::RotaryTable table;
};

namespace sa {
namespace {

constexpr int kThreads = 256;

struct RotaryArgs {
  const uint16_t *q, *k;
  uint16_t *qo, *ko;
  int64_t q_hs, q_rs, k_hs, k_rs, qo_hs, qo_rs, ko_hs, ko_rs;
  const int32_t *positions;
  int64_t pos;
  int n, Hq, H;     // query heads, heads of both sides
  int per;          // heads of a thread
  int pairs, copy;  // rotary_dim / 2; whether the elements behind the pairs are written
  RotaryTable f;
};

template <int W> struct Vec;
template <> struct Vec<4> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <> struct Vec<2> { typedef uint32_t type; };
template <> struct Vec<1> { typedef uint16_t type; };

template <int W>
union Chunk {
  typename Vec<W>::type v;
  uint16_t e[W];
};

__device__ inline float value(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ inline uint16_t rounded(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// A row is cut into 64 / W units of 2W elements: those of the pairs first (the two halves' W elements, or 2W
// neighbours), then those that pass.  W divides the number of pairs, so that a unit is all pairs or none and its two
// accesses are aligned.  256 threads: units of consecutive tokens.
template <int W, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs p) {
  constexpr int kUnits = 64 / W, kTokens = kThreads / kUnits;
  const int u = threadIdx.x % kUnits;
  const int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / kUnits;
  if (t >= p.n) return;
  const bool turns = u * W < p.pairs;
  if (!turns && !p.copy) return;
  const int h0 = blockIdx.y * p.per, h1 = min(h0 + p.per, p.H);
  const int a = turns && HALF ? u * W : 2 * u * W;   // first element of either access
  const int b = turns && HALF ? a + p.pairs : a + W;
  Chunk<W> xa, xb;
  auto read = [&](int h) {
    const uint16_t *x = h < p.Hq ? p.q + h * p.q_hs + t * p.q_rs : p.k + (h - p.Hq) * p.k_hs + t * p.k_rs;
    xa.v = *(const typename Vec<W>::type *)(x + a);
    xb.v = *(const typename Vec<W>::type *)(x + b);
  };
  read(h0);  // on its way while the sines are taken
  float c[W], s[W];
  if (turns) {
    const uint64_t at = (uint64_t)(p.positions ? (int64_t)p.positions[t] : p.pos + t);
#pragma unroll
    for (int e = 0; e < W; ++e) {
      const uint64_t turn = at * p.f.turn[u * W + e];
      // the nearest multiple of 2^-32 of a turn, in [-1/2, 1/2), and sine and cosine of pi times twice that
      const float x = (float)(int32_t)((turn + 0x80000000ull) >> 32) * 0x1p-31f;
      sincospif(x, &s[e], &c[e]);
      s[e] *= p.f.sine;
      c[e] *= p.f.cosine;
    }
  }
  for (int h = h0; h < h1; ++h) {
    if (h > h0) read(h);
    uint16_t *y = h < p.Hq ? p.qo + h * p.qo_hs + t * p.qo_rs : p.ko + (h - p.Hq) * p.ko_hs + t * p.ko_rs;
    if (turns) {
      if (HALF) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float r = value(xa.e[e]), i = value(xb.e[e]);
          xa.e[e] = rounded(r * c[e] - i * s[e]);
          xb.e[e] = rounded(r * s[e] + i * c[e]);
        }
      } else {
        uint16_t z[2 * W];
#pragma unroll
        for (int e = 0; e < W; ++e) { z[e] = xa.e[e]; z[W + e] = xb.e[e]; }
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const float r = value(z[2 * e]), i = value(z[2 * e + 1]);
          z[2 * e] = rounded(r * c[e] - i * s[e]);
          z[2 * e + 1] = rounded(r * s[e] + i * c[e]);
        }
#pragma unroll
        for (int e = 0; e < W; ++e) { xa.e[e] = z[e]; xb.e[e] = z[W + e]; }
      }
    }
    typename Vec<W>::type *ya = (typename Vec<W>::type *)(y + a), *yb = (typename Vec<W>::type *)(y + b);
    if constexpr (W == 4) {  // many rows: outputs that the caches need not keep, see below
      __builtin_nontemporal_store(xa.v, ya);
      __builtin_nontemporal_store(xb.v, yb);
    } else {
      *ya = xa.v;
      *yb = xb.v;
    }
  }
}

template <int W>
void launch(const RotaryArgs &a, bool half, dim3 grid, hipStream_t st) {
  if (half) rotary_kernel<W, true><<<grid, kThreads, 0, st>>>(a);
  else rotary_kernel<W, false><<<grid, kThreads, 0, st>>>(a);
}

// Frequencies in turns per position, as fractions of 2^64.  They are taken modulo one turn, which a position's
// product does not see.
bool make_table(const sa_rotary_config &c, RotaryTable *t) {
  const int dim = c.rotary_dim;
  const long double two_pi = 6.283185307179586476925286766559L;
  long double theta = c.theta;
  if (c.scaling == SA_SCALING_BASE && dim > 2) theta *= powl(c.factor, (long double)dim / (dim - 2));
  long double lo = 0, hi = 0;
  if (c.scaling == SA_SCALING_RAMP) {
    auto turning = [&](double r) { return dim * logl(c.original_len / (two_pi * r)) / (2 * logl(theta)); };
    lo = fmaxl(floorl(turning(c.high)), 0);
    hi = fminl(ceill(turning(c.low)), dim - 1);
  }
  for (int i = 0; i < dim / 2; ++i) {
    long double w = powl(theta, -2.0L * i / dim);
    if (c.scaling == SA_SCALING_LINEAR) w /= c.factor;
    if (c.scaling == SA_SCALING_WAVELENGTH) {
      const long double k = fminl(fmaxl((c.original_len * w / two_pi - c.low) / ((long double)c.high - c.low), 0), 1);
      w = k * w + (1 - k) * w / c.factor;
    }
    if (c.scaling == SA_SCALING_RAMP) {
      const long double k = fminl(fmaxl((i - lo) / fmaxl(hi - lo, 0.001L), 0), 1);
      w = (1 - k) * w + k * w / c.factor;
    }
    const long double turns = w / two_pi;  // < 1: theta > 1 and factor >= 1
    if (!(turns >= 0 && turns < 1)) return false;
    t->turn[i] = (uint64_t)(turns * 0x1p64L);
  }
  for (int i = dim / 2; i < 64; ++i) t->turn[i] = 0;
  t->cosine = (float)c.amplitude;
  t->sine = (float)(c.transposed ? -c.amplitude : c.amplitude);
  t->pairs = dim / 2;
  t->layout = c.layout;
  return true;
}

}  // namespace

const RotaryTable &rotary_table(const sa_rotary *r) { return r->table; }

hipError_t launch_rotary(const Shape &sh, const RotaryTable &f, sa_rows Q, sa_rows K, int64_t n, int64_t pos,
                         const int32_t *positions, sa_rows Qo, sa_rows Ko, hipStream_t st) {
  RotaryArgs a;
  a.q = (const uint16_t *)Q.data; a.k = (const uint16_t *)K.data;
  a.qo = (uint16_t *)Qo.data; a.ko = (uint16_t *)Ko.data;
  a.q_hs = Q.head_stride; a.q_rs = Q.row_stride; a.k_hs = K.head_stride; a.k_rs = K.row_stride;
  a.qo_hs = Qo.head_stride; a.qo_rs = Qo.row_stride; a.ko_hs = Ko.head_stride; a.ko_rs = Ko.row_stride;
  a.positions = positions; a.pos = pos; a.n = (int)n;
  a.Hq = Q.data ? sh.Hq : 0;
  a.H = a.Hq + (K.data ? sh.Hkv : 0);
  a.pairs = f.pairs;
  a.copy = (Q.data && Q.data != Qo.data) || (K.data && K.data != Ko.data);
  a.f = f;
  // The widest W of 4, 2 and 1 that divides the pairs; 2 at most where there are few rows, for shorter chains of sines
  // (1 token of 40 heads 2.2 us instead of 2.6, 300 tokens 3.8 instead of 3.4).  8 is slower: 10304 tokens 43 us instead of 40.
  // Outputs of many rows, 1 MB and more, go past the caches (10304 tokens 40 -> 37 us).
  const int most = n * a.H <= 4096 ? 2 : 4;
  const int w = most >= 4 && f.pairs % 4 == 0 ? 4 : f.pairs % 2 == 0 ? 2 : 1;
  const int64_t tiles = (n + kThreads * w / 64 - 1) / (kThreads * w / 64);
  // Heads of a thread: as many as leave eight workgroups a compute unit, but three at most.  With more the workgroups, which
  // drift apart, have every head's memory open at once: 128K tokens of 40 heads (2.68 GB) in a replayed loop 429 us with 3 heads,
  // 479 with 16 and 508 with all 40; one head each costs the sines, 555.
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(a.H, 8 * (int64_t)sh.n_cu / tiles));
  a.per = std::min((int)((a.H + want - 1) / want), 3);
  const dim3 grid((unsigned)tiles, (unsigned)((a.H + a.per - 1) / a.per));
  const bool half = f.layout == SA_ROTARY_HALF;
  switch (w) {
    case 4: launch<4>(a, half, grid, st); break;
    case 2: launch<2>(a, half, grid, st); break;
    default: launch<1>(a, half, grid, st);
  }
  return hipGetLastError();
}

}  // namespace sa

extern "C" {

sa_status sa_rotary_create(const sa_rotary_config *cfg, sa_rotary **out) {
  if (!cfg || !out) return SA_ERR_INVALID_ARG;
  *out = nullptr;
  sa_rotary_config c = *cfg;
  if (c.rotary_dim == 0) c.rotary_dim = sa::kHeadDim;
  if (c.theta == 0) c.theta = 10000;
  if (c.rotary_dim < 2 || c.rotary_dim % 2 || c.rotary_dim > sa::kHeadDim) return SA_ERR_UNSUPPORTED;
  if (c.layout != SA_ROTARY_HALF && c.layout != SA_ROTARY_INTERLEAVED) return SA_ERR_INVALID_ARG;
  if (c.scaling < SA_SCALING_NONE || c.scaling > SA_SCALING_RAMP) return SA_ERR_INVALID_ARG;
  if (c.transposed != 0 && c.transposed != 1) return SA_ERR_INVALID_ARG;
  if (!(c.theta > 1) || !std::isfinite(c.theta)) return SA_ERR_INVALID_ARG;
  if (c.scaling != SA_SCALING_NONE && (!(c.factor >= 1) || !std::isfinite(c.factor))) return SA_ERR_INVALID_ARG;
  if (c.scaling == SA_SCALING_WAVELENGTH || c.scaling == SA_SCALING_RAMP)
    if (!(c.low > 0) || !(c.high > c.low) || !(c.original_len > 0) || !std::isfinite(c.high) || !std::isfinite(c.original_len))
      return SA_ERR_INVALID_ARG;
  if (c.amplitude == 0) c.amplitude = c.scaling == SA_SCALING_RAMP ? 0.1 * std::log(c.factor) + 1 : 1;
  if (!(c.amplitude > 0) || !std::isfinite((float)c.amplitude)) return SA_ERR_INVALID_ARG;
  sa_rotary *r = new (std::nothrow) sa_rotary();
  if (!r) return SA_ERR_INVALID_ARG;
  r->cfg = c;
  if (!sa::make_table(c, &r->table)) { delete r; return SA_ERR_INVALID_ARG; }
  *out = r;
  return SA_OK;
}

void sa_rotary_destroy(sa_rotary *r) { delete r; }

}  // extern "C"
