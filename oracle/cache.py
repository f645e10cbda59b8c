"""fp64 oracle of the 8-bit key/value cache: what a block's codes and scale are, and what they stand for.  TEST
INFRASTRUCTURE ONLY."""
from __future__ import annotations

import numpy as np

E4M3, E5M2 = 0, 1
LARGEST = (448.0, 57344.0)


def values(kind):
    """The 256 values of a type by code (OCP 8-bit floating point)."""
    bits, bias = ((3, 7), (2, 15))[kind]
    out = np.empty(256)
    for code in range(256):
        e, f = (code & 0x7F) >> bits, code & ((1 << bits) - 1)
        v = (1 + f / 2 ** bits) * 2.0 ** (e - bias) if e else f / 2 ** bits * 2.0 ** (1 - bias)
        if kind == E4M3 and (code & 0x7F) == 0x7F:
            v = np.nan
        if kind == E5M2 and e == 31:
            v = np.nan if f else np.inf
        out[code] = -v if code & 0x80 else v
    return out


def scale(block, kind):
    """The scale of a block of values (fp64)."""
    finite = np.abs(block[np.isfinite(block)])
    top = finite.max() if finite.size else 0.0
    if top == 0:
        return 1.0
    e = -100
    while 2.0 ** e * LARGEST[kind] < top:
        e += 1
    return 2.0 ** e


def nearest(x, kind):
    """The values of the type nearest to x, ties to the even code; NaN stays, infinities as the type has them."""
    v = values(kind)[:128]
    order = np.arange(0x7F if kind == E4M3 else 0x7C)  # finite codes, ascending
    v = v[order]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(v, np.where(np.isfinite(a), a, 0)), 1, len(v) - 1)
    lo = hi - 1
    below, above = np.where(np.isfinite(a), a, 0) - v[lo], v[hi] - np.where(np.isfinite(a), a, 0)
    pick = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    y = np.copysign(v[pick], x)
    y = np.where(np.isnan(x), np.nan, y)
    return np.where(np.isinf(x), np.copysign(np.inf, x) if kind == E5M2 else np.nan, y)


def contents(x, block, kind):
    """Of x [heads, tokens, 128] fp64: codes as values [heads, full, 128], scales [heads, full / block], the open rows."""
    heads, tokens, _ = x.shape
    full = tokens // block * block
    codes, scales = np.empty((heads, full, x.shape[2])), np.empty((heads, full // block))
    for h in range(heads):
        for b in range(full // block):
            part = x[h, b * block:(b + 1) * block]
            scales[h, b] = scale(part, kind)
            codes[h, b * block:(b + 1) * block] = nearest(part / scales[h, b], kind)
    return codes, scales, x[:, full:]


def read(x, block, kind):
    """What a reader of the cache sees of x."""
    codes, scales, rest = contents(x, block, kind)
    return np.concatenate([codes * np.repeat(scales, block, 1)[..., None], rest], 1)
