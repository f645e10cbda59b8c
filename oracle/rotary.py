"""fp64 oracle of the rotary positions: angles in long double, the rotation in fp64.  TEST INFRASTRUCTURE ONLY."""
from __future__ import annotations

import math

import numpy as np

NONE, LINEAR, BASE, WAVELENGTH, RAMP = range(5)


def frequencies(dim, theta=10000.0, scaling=NONE, factor=1.0, low=1.0, high=4.0, original_len=8192.0):
    """Radians per position of the pairs of the first `dim` elements."""
    L = np.longdouble
    w = []
    for i in range(dim // 2):
        base = L(theta)
        if scaling == BASE and dim > 2:
            base = base * L(factor) ** (L(dim) / (dim - 2))
        f = base ** (L(-2 * i) / dim)
        if scaling == LINEAR:
            f = f / factor
        elif scaling == WAVELENGTH:
            turns = float(f) * original_len / (2 * math.pi)   # in the original length
            if turns < low:
                f = f / factor
            elif turns < high:
                t = (L(original_len) * f / (2 * np.arccos(L(-1))) - low) / (L(high) - low)
                f = (1 - t) * f / factor + t * f
        elif scaling == RAMP:
            def pair(r):
                return dim * math.log(original_len / (r * 2 * math.pi)) / (2 * math.log(theta))
            a, b = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), dim - 1)
            t = min(max((L(i) - a) / max(L(b - a), L(0.001)), L(0)), L(1))
            f = f * (1 - t) + f / factor * t
        w.append(f)
    return np.array(w, np.longdouble)


def amplitude(scaling=NONE, factor=1.0, given=0.0):
    return given if given else (0.1 * math.log(factor) + 1.0 if scaling == RAMP else 1.0)


def rotate(x, positions, w, interleaved=False, transposed=False, amp=1.0):
    """x [heads, n, 128] fp64, positions [n] integers, w from frequencies()."""
    half = len(w)
    turns = np.asarray(positions, np.int64)[:, None].astype(np.longdouble) * w / (2 * np.arccos(np.longdouble(-1)))
    angle = ((turns - np.rint(turns)) * (2 * np.arccos(np.longdouble(-1)))).astype(np.float64)
    c, s = amp * np.cos(angle), amp * np.sin(angle) * (-1 if transposed else 1)
    y = np.array(x, np.float64)
    at = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    return y
