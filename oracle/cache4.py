"""fp64 oracle of the 4-bit key/value cache: what a group's codes and scale are, and what they stand for.  TEST INFRASTRUCTURE
ONLY."""
from __future__ import annotations

import numpy as np

GROUP = 32
VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])  # OCP e2m1, by code


def exponents(x):
    """Scale exponents of groups [..., 32], NaN where a value is not finite."""
    top = np.abs(np.where(np.isfinite(x), x, 0)).max(-1)
    e = np.full(top.shape, -100.0)
    for k in range(-100, 125):
        e[top >= 7 * 2.0 ** k] = k + 1
    e[top == 0] = 0
    return np.where(np.isfinite(x).all(-1), e, np.nan)


def nearest(y):
    """Codes of the values nearest to y, ties to the even code; 6 behind it."""
    a = np.minimum(np.abs(y), 6.0)
    hi = np.clip(np.searchsorted(VALUES[:8], a), 1, 7)
    lo = hi - 1
    below, above = a - VALUES[lo], VALUES[hi] - a
    pick = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    return (pick + 8 * np.signbit(y)).astype(np.uint8)


def contents(x):
    """Of x [heads, tokens, 128] fp64: packed codes [heads, tokens, 64] and scale bytes [heads, tokens, 4]."""
    g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    e = exponents(g)
    number = ~np.isnan(e)
    codes = nearest(np.where(number[..., None], g, 0) / 2.0 ** np.where(number, e, 0)[..., None])
    codes = np.where(number[..., None], codes, 0).astype(np.uint8).reshape(x.shape)
    return codes[..., 0::2] | codes[..., 1::2] << 4, np.where(number, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    """What packed codes and scale bytes stand for."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1, GROUP)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (VALUES[c] * s[..., None]).reshape(*codes.shape[:-1], -1)


def read(x):
    """What a reader of the cache sees of x."""
    return values(*contents(x))


E2M3 = np.array([(1 + m / 8) * 2.0 ** (e - 1) if e else m / 8 for e in range(4) for m in range(8)])  # OCP e2m3 magnitudes, by code


def _bf16(x):
    """fp32 values rounded to bf16, ties to even."""
    bits = x.astype(np.float32).view(np.uint32)
    return ((bits + 0x7FFF + ((bits >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32).astype(np.float64)


def query_left_out(q, c=1.0):
    """What three e2m3 codes of the elements of q [..., 128] times c in fp32 (scales 2^e, 2^(e - 4), 2^(e - 8) of a group of 32, the least
    e >= -118 with every magnitude <= 7.5 * 2^e; a code is the nearest to what is left, rounded to bf16 first) leave of them."""
    r = (q.astype(np.float32) * np.float32(c)).astype(np.float64).reshape(*q.shape[:-1], -1, GROUP)
    top = np.abs(r).max(-1)
    m, e = np.frexp(top / 7.5)  # top = 7.5 m 2^e, m in [0.5, 1)
    s = 2.0 ** np.where(top > 0, np.maximum(e - (m == 0.5), -118), -118)[..., None]
    for k in range(3):
        unit = s * 2.0 ** (-4 * k)
        a = np.minimum(np.abs(_bf16(r)) / unit, 7.5)
        hi = np.clip(np.searchsorted(E2M3, a), 1, 31)
        below, above = a - E2M3[hi - 1], E2M3[hi] - a
        r = r - np.copysign(E2M3[np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, hi - 1)] * unit, r)
    return r.reshape(q.shape)
