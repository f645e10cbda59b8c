"""Pins of the 4-bit cache's oracle by hand-made groups and by what its definition says (no GPU needed)."""
import numpy as np
import pytest

from oracle import cache4 as oc


def _group(*head):
    x = np.zeros((1, 1, 128))
    x[0, 0, :len(head)] = head
    return x


def test_codes_of_every_middle_and_value():
    y = np.array([0, 0.2, 0.25, 0.26, 0.5, 0.74, 0.75, 0.76, 1, 1.25, 1.3, 1.5, 1.74, 1.75, 2, 2.5, 2.6, 3, 3.4, 3.5, 4, 5, 5.1, 6, 6.9])
    want = [0, 0, 0, 1, 1, 1, 2, 2, 2, 2, 3, 3, 3, 4, 4, 4, 5, 5, 5, 6, 6, 6, 7, 7, 7]
    assert oc.nearest(y).tolist() == want
    assert oc.nearest(-y).tolist() == [w + 8 for w in want]


@pytest.mark.parametrize("top,e", [(6.0, 0), (6.97, 0), (7.0, 1), (13.9, 1), (14.0, 2), (3.49, -1), (3.5, 0), (1e-40, -100),
                                   (7 * 2.0 ** -100, -99), (2.0 ** 127, 125), (1.99 * 2.0 ** 127, 125), (1.7 * 2.0 ** 127, 125)])
def test_scales(top, e):
    codes, scales = oc.contents(_group(-top, top / 3))
    assert scales[0, 0].tolist() == [e + 127, 127, 127, 127]
    back = oc.values(codes, scales)[0, 0]
    assert np.abs(back[0] + top) <= (2.0 ** e if top < 7 * 2.0 ** 125 else 2.0 ** 126)  # half the widest step, or saturated


def test_packing_and_zeros():
    codes, scales = oc.contents(_group(1.0, -1.5, 6.0, -0.0))
    assert codes[0, 0, :2].tolist() == [2 | 11 << 4, 7 | 8 << 4] and not codes[0, 0, 2:].any()
    assert np.array_equal(oc.values(codes, scales)[0, 0, :4], [1.0, -1.5, 6.0, 0.0])


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_groups_that_are_no_numbers(bad):
    x = np.ones((2, 3, 128))
    x[1, 2, 40] = bad
    codes, scales = oc.contents(x)
    assert scales[1, 2].tolist() == [125, 255, 125, 125] and (codes[1, 2, 16:32] == 0).all()
    back = oc.values(codes, scales)
    assert np.isnan(back[1, 2, 32:64]).all() and np.isfinite(back).sum() == back.size - 32


def test_no_value_is_off_by_more_than_half_a_step():
    x = np.random.default_rng(1).standard_normal((4, 50, 128)) * 2.0 ** np.random.default_rng(2).integers(-20, 20, (4, 50, 1))
    back, (_, scales) = oc.read(x), oc.contents(x)
    s = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    step = np.where(np.abs(x) < 2 * s, 0.5, np.where(np.abs(x) < 4 * s, 1.0, 2.0)) * s
    assert (np.abs(back - x) <= step / 2).all()
    top = np.abs(x.reshape(4, 50, 4, 32)).max(-1)
    assert (top < 7 * 2.0 ** (scales.astype(float) - 127)).all() and (top >= 3.5 * 2.0 ** (scales.astype(float) - 127)).all()


def test_three_codes_of_a_query():
    # every finite bf16 value beside a largest one of its group, times softmax scales.  A code is off by half its step, and by what bf16 rounded before it
    # was chosen (2^-9 of it): of the first code's scale s at most 0.25 + 2^-6, so the second stays below 4.3 of its own and is off by 0.25 + 2^-6, or
    # 0.125 + 2^-7 below 4, where it nearly always is; the third, again below 4.3, by 0.125 + 2^-7 up to 4 and 0.27 behind.  0.27 * 2^-8 s needs both
    # ends at once; what is there is held by 2^-10.9 s, 2^-12.8 of the largest.  Without a factor, 8 bits: 2^-12 s, and nothing from a
    # 16th of s on.
    from harness import gen

    x = gen.bf16_bits_to_f32(np.arange(65536, dtype=np.uint16)).astype(np.float64)
    for top in (7.5, 4.0, 3.78125, 1.0, 2.0 ** 20, 1.984375 * 2.0 ** 110):
        y = x[np.abs(x) <= top]
        y = np.concatenate([y, np.zeros(-len(y) % 31)]).reshape(-1, 31)
        q = np.concatenate([np.full((len(y), 1), top), y], 1)
        q = np.concatenate([q, np.zeros((-len(q) % 4, 32))]).reshape(-1, 128)
        for c in (1.0, 128.0 ** -0.5 * 1.4426950408889634, 0.02, 1.9):
            left = np.abs(oc.query_left_out(q, c))
            largest = top * np.float32(c)
            s = 2.0 ** np.ceil(np.log2(largest / 7.5))
            if c == 1.0:
                assert left.max() <= s * 2.0 ** -12, (top, left.max() / s)
                assert not left[np.abs(q) >= s / 16].any(), (top, np.abs(q)[left > 0].max() / s)
            assert left.max() <= s * 2.0 ** -10.9 and left.max() <= largest * 2.0 ** -12.8
    assert not oc.query_left_out(np.zeros((1, 128))).any()
