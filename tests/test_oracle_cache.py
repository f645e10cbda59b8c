"""The oracles of the rotary positions and of the 8-bit cache against properties that define them."""
import numpy as np
import pytest

from oracle import cache as oc
from oracle import rotary as orot


@pytest.mark.parametrize("kind,largest,least,codes", [(oc.E4M3, 448.0, 2.0 ** -9, 254), (oc.E5M2, 57344.0, 2.0 ** -16, 248)])
def test_values_of_the_types(kind, largest, least, codes):
    v = oc.values(kind)
    f = v[np.isfinite(v)]
    assert len(f) == codes and f.max() == largest == oc.LARGEST[kind] and f[f > 0].min() == least
    assert (np.sort(v[:128][np.isfinite(v[:128])]) == v[:128][np.isfinite(v[:128])]).all()
    assert (oc.nearest(f, kind) == f).all()


@pytest.mark.parametrize("kind", [oc.E4M3, oc.E5M2])
def test_nearest_is_nearest_and_even(kind):
    rng = np.random.default_rng(1)
    x = rng.uniform(-1, 1, 4000) * oc.LARGEST[kind] * 2.0 ** rng.integers(-24, 1, 4000)
    v = oc.values(kind)
    f = v[np.isfinite(v)]
    assert (np.abs(oc.nearest(x, kind) - x) == np.abs(f[None] - x[:, None]).min(1)).all()
    pos = v[:128][np.isfinite(v[:128])]
    mid = (pos[1:] + pos[:-1]) / 2  # ties go to the even code
    want = np.where(np.arange(len(mid)) % 2 == 0, pos[:-1], pos[1:])
    assert (oc.nearest(mid, kind) == want).all() and (oc.nearest(-mid, kind) == -want).all()


@pytest.mark.parametrize("kind", [oc.E4M3, oc.E5M2])
def test_scale_is_the_least_power_of_two(kind):
    top = oc.LARGEST[kind]
    for a, want in [(top, 1.0), (np.nextafter(top, 1e9), 2.0), (top / 2, 0.5), (0.0, 1.0), (2.0 ** -130, 2.0 ** -100), (np.inf, 1.0)]:
        assert oc.scale(np.array([0.0, -a]), kind) == want


def test_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((1, 6, 128))
    w = orot.frequencies(128)
    for interleaved in (False, True):
        y = orot.rotate(x, [0, 1, 2, 1000, 131072, 2 ** 31 - 1], w, interleaved)
        assert np.allclose(np.linalg.norm(x, axis=-1), np.linalg.norm(y, axis=-1), rtol=1e-13)
        assert np.allclose(y[:, 0], x[:, 0])
        back = orot.rotate(y, [0, 1, 2, 1000, 131072, 2 ** 31 - 1], w, interleaved, transposed=True)
        assert np.allclose(back, x, atol=1e-13)
        # the product of a rotated query and key depends on their distance alone
        q, k = x[:, :1], x[:, 1:2]
        dots = [(orot.rotate(q, [p + 7], w, interleaved) * orot.rotate(k, [p], w, interleaved)).sum() for p in (0, 5, 100000)]
        assert np.ptp(dots) < 1e-9


def test_scalings():
    plain = orot.frequencies(64)
    assert np.allclose(orot.frequencies(64, scaling=orot.LINEAR, factor=4.0) * 4, plain)
    base = orot.frequencies(64, scaling=orot.BASE, factor=8.0)
    assert base[0] == plain[0] and np.isclose(float(base[-1]) * 8, float(plain[-1]))  # the slowest pair by the whole factor
    for s, more in ((orot.WAVELENGTH, dict(low=1.0, high=4.0)), (orot.RAMP, dict(low=1.0, high=32.0))):
        f = orot.frequencies(128, theta=500000.0, scaling=s, factor=8.0, original_len=8192.0, **more)
        p = orot.frequencies(128, theta=500000.0)
        r = (p / f).astype(float)
        assert r[0] == 1 and np.isclose(r[-1], 8) and (np.diff(r) >= -1e-12).all()
