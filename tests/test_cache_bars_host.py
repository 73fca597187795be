"""The bars of cache_attention's results (cache_bars.py) tell, from what they allow, weights of 16 bits in place of 23 (few
queries), a lost second part of the weights (many queries), and codes cut instead of rounded. The mistakes are planted in
the 64-bit definition."""
import numpy as np
import pytest

import attention_bars
import cache_bars as bars

LARGEST = 8355000.0


def digits(w):
    """w as the whole number that stands for it."""
    return np.rint(w * LARGEST) / LARGEST


def two_digits(w):
    """The lowest of its three signed digits to the base 256 lost."""
    return np.floor((np.rint(w * LARGEST) + 128) / 256) * 256 / LARGEST


def cut(w, bits):
    m, e = np.frexp(w)
    return np.ldexp(np.floor(np.ldexp(m, bits)), e - bits)


def half(w):
    """w cut to a 16-bit float."""
    return np.where(w < 2.0 ** -14, np.floor(w * 2.0 ** 24) * 2.0 ** -24, cut(w, 11))


def one_part(w):
    return half(w * 2.0 ** 7) * 2.0 ** -7


def two_parts(w):
    p = w * 2.0 ** 7
    return (half(p) + half(p - half(p))) * 2.0 ** -7


FORMS = {"split": (digits, two_digits), "prompt": (two_parts, one_part)}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("news,lens", [([3, 2, 1], [15, 3, 1]), ([4, 1], [64, 33]), ([8, 8], [200, 130]), ([6], [700]),
                                       ([3], [2000])])
@pytest.mark.parametrize("nh,nkv,hd", [(2, 2, 64), (8, 2, 128), (6, 1, 48), (12, 12, 16)])
def test_what_is_lost_is_seen(form, news, lens, nh, nkv, hd):
    rng = np.random.default_rng([sum(lens), nh, hd])
    codes = lambda *shape: np.clip(np.rint(rng.standard_normal(shape) * 32), -127, 127).astype(np.int8)  # noqa: E731
    ps = 16
    count = [-(-n // ps) for n in lens]
    table = np.full((len(lens), max(count)), -1, np.int32)
    for s, c in enumerate(count):
        table[s, :c] = np.arange(c) + sum(count[:s])
    cache, q = codes(sum(count), 2, nkv, ps, hd), codes(sum(news), nh * hd)
    start = np.concatenate([[0], np.cumsum(news)])

    def run(weights):
        return bars.attention(q, cache, start, lens, table, nh, 0.04 * 0.05 * hd ** -0.5, True, form, weights=weights)

    want, bar, real = run(lambda w: w)
    assert real.all() and bar.max() <= 127 * 4e-5
    so = attention_bars.output_scale(want)
    good, bad = (run(f)[0] for f in FORMS[form])
    for y in (want, good):
        attention_bars.assert_within(y, want, bar)
        attention_bars.assert_within(np.rint(y / so), want, bar, so)
    with pytest.raises(AssertionError):
        attention_bars.assert_within(bad, want, bar)
    with pytest.raises(AssertionError):
        attention_bars.assert_within(np.trunc(want / so), want, bar, so)
