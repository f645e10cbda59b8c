"""How near two codes of e4m3 come to a bf16 element of a query, by all of its values: the 128-row attention over the cache multiplies
q = hi + lo, hi the code nearest to q / s, lo the one nearest to 16 (q / s - hi), with the least power of two s that brings the
row's largest element to 448 s or below, so into (224 s, 448 s]."""
import numpy as np

from oracle import cache as oc


def _split(x):
    hi = oc.nearest(x, oc.E4M3)
    return hi, oc.nearest(16 * (x - hi), oc.E4M3) / 16


def _elements(low):
    """Every bf16 magnitude from 2^low to 448."""
    x = (1 + np.arange(128) / 128) * 2.0 ** np.arange(low, 9)[:, None]
    return x[x <= 448]


def test_exact_from_a_14th_binary_place_on():
    x = _elements(-6)
    hi, lo = _split(x)
    assert (hi + lo == x).all() and (np.abs(lo) <= 448).all()
    hi, lo = _split(-x)
    assert (hi + lo == -x).all()


def test_what_smaller_elements_lose():
    x = _elements(-60)
    hi, lo = _split(x)
    off = np.abs(x - hi - lo)
    assert off.max() == 2.0 ** -14                   # half a step of the least codes, a 16th of them
    assert off.max() / 224 < 2.0 ** -21.8            # of the row's largest element at most
    assert off[x >= 2.0 ** -6].max() == 0 and 2.0 ** -6 / 224 < 2.0 ** -13.8
    assert _split(np.array([2.0 ** -14])) == (0, 0)  # the whole element
