"""The bars of attention results tell a lost second part of the softmax weights, and
codes cut instead of rounded, from what they allow. Both mistakes are planted in the
64-bit definition."""
import numpy as np
import pytest

import attention_bars as bars


def cut(w, bits):
    """w cut to that many significant bits."""
    m, e = np.frexp(w)
    return np.ldexp(np.floor(np.ldexp(m, bits)), e - bits)


def one_part(w):
    return cut(w * 2.0 ** 7, 11) * 2.0 ** -7


def two_parts(w):
    """The first part, and the remainder as a 16-bit float (step 2^-24 at its smallest)."""
    p = w * 2.0 ** 7
    first = cut(p, 11)
    return (first + (p - first).astype(np.float16).astype(np.float64)) * 2.0 ** -7


CASES = [([128] * 8, 4, 64), ([384, 384, 100], 2, 64), ([300, 1, 77], 3, 128), ([200, 16], 4, 16), ([1000], 2, 64)]


def run(lens, nh, hd, weights):
    x = bars.codes(np.random.default_rng([sum(lens), nh, hd]), sum(lens), 3 * nh * hd)
    xs = float(np.float32(0.04))
    return bars.attention(x, xs, bars.starts(lens), nh, nh, hd, hd ** -0.5, weights=weights)


@pytest.mark.parametrize("lens,nh,hd", CASES)
def test_a_lost_second_part_is_seen(lens, nh, hd):
    want, bar = run(lens, nh, hd, lambda w: w)
    so = bars.output_scale(want)
    for good in (want, run(lens, nh, hd, two_parts)[0]):
        bars.assert_within(good.astype(np.float32), want, bar)
        bars.assert_within(np.rint(good / so), want, bar, so)
    bad = run(lens, nh, hd, one_part)[0]
    with pytest.raises(AssertionError):
        bars.assert_within(np.rint(bad / so), want, bar, so)
    with pytest.raises(AssertionError):
        bars.assert_within(bad.astype(np.float32), want, bar)
    with pytest.raises(AssertionError):
        bars.assert_within(np.trunc(want / so), want, bar, so)
    # (a bar of half a step and 2^-10 of the largest value, as for one part, would not have seen it)
    assert np.abs(np.rint(bad / so) - want / so).max() <= 0.5 + 2 * 2.0 ** -10 * 128 * 0.04 / so
