"""How far results of attention_run may be from their definition in 64 bits, and
the definition with what these bars need. Shares no code with the library.

For a query, with w_j = 2^(E_j) the weights relative to the largest (E_j <= 0, E
the largest |E_j|), n the keys that take part, and A = sum_j w_j |v_j| / sum_j w_j
for every feature:

* The exponent's factor is held in 22 bits: |E| 2^-22 of an exponent. Its product
  with the score is rounded once, and so is the exponential (2^-23): together at
  most 2^-23 + (E + 16) 2^-22 of a weight.
* A weight enters the products in two 16-bit parts. The first is its value cut to
  11 bits, the second the remainder rounded to 11: 2^-21 of the weight at most.
  16-bit floats end at a step of 2^-24, and weights carry a factor of 2^7: below
  2^-10 of the largest, an absolute error of up to `step` = 2^-31 of the largest
  comes in its place.
* The sum of weights is that of the values before the cut.
* O is summed in fp32, two products for 16 keys, each of which may round 2 times:
  n / 4 roundings of 2^-24 of A; the sum of weights n / 64 + 32.

An error d of the weights moves their mean by 2 d A. An int8 code lies within half
a step and that of its value; codes that differ from the rounded definition are
those whose value lies that near to a half. With one 16-bit part alone 0.4 % of the
codes of 128-token sequences differ; an eighth of that is allowed.
"""
import numpy as np

import encoder_ref as ref

STEP = 2.0 ** -31


def attention(x, x_scale, start, nh, nkv, hd, softmax_scale, key_len=None, lists=None, query_block=64, step=STEP,
              weights=lambda w: w):
    """y [M, nh * hd] in float64 and its bar, for valid keys and lists of different blocks as attention_run takes them.
    `weights`: applied to the weights that meet v, not to those summed."""
    y, bar = np.zeros((len(x), nh, hd)), np.zeros((len(x), nh, hd))
    for s in range(len(start) - 1):
        q, k, v = ref.split_heads(x, start, s, nh, nkv, hd, key_len)
        n, keys = len(q), len(k)
        if n == 0 or keys == 0:
            continue
        for h in range(nh):
            kv = h // (nh // nkv)
            z = q[:, h] @ k[:, kv].T * (float(x_scale) ** 2 * softmax_scale * np.log2(np.e))
            use = np.ones((n, keys), bool) if lists is None else ref.listed(lists[s, h], n, keys, query_block)
            some = use.any(1)
            top = np.where(some, np.where(use, z, -np.inf).max(1), 0.0)
            spread = np.where(some, top - np.where(use, z, np.inf).min(1), 0.0)
            w = np.where(use, np.exp2(np.minimum(z - top[:, None], 0.0)), 0.0)
            total = np.where(some, w.sum(1), 1.0)[:, None]
            count = use.sum(1)[:, None]
            vj, mag = v[:, kv] * x_scale, np.abs(v[:, kv]) * x_scale
            a = w @ mag / total
            rel = 2.0 ** -23 + (spread[:, None] + 16) * 2.0 ** -22 + 2.0 ** -21
            rounded = (count / 4 + count / 64 + 32) * 2.0 ** -24
            y[start[s]:start[s + 1], h] = weights(w) @ vj / total
            bar[start[s]:start[s + 1], h] = (2 * rel + rounded) * a + step * (use @ mag) / total
    return y.reshape(len(x), -1), bar.reshape(len(x), -1)


def output_scale(want):
    return float(np.float32(max(np.abs(want).max(initial=0.0), 1e-3) / 126))


def assert_within(got, want, bar, out_scale=None):
    """Asserts that fp32 results, or int8 codes of out_scale, are within the bars."""
    if got.size == 0:
        return
    if out_scale is None:
        over = np.abs(got.astype(np.float64) - want) - bar
        assert np.isfinite(got).all() and over.max() <= 0, f"{over.max()} over the bar"
        return
    z = np.clip(want / out_scale, -127, 127)
    tie = 4 * 128 * 2.0 ** -24  # the conversion to codes: a division and two products in fp32, on at most 127
    over = np.abs(got - z) - (0.5 + bar / out_scale + tie)
    assert over.max() <= 0, f"codes: {over.max()} over the bar"
    # (a value that is a half to within the conversion has two right codes; where many queries see one key, all are it)
    differ = int(((got != np.rint(z)) & (np.abs(np.abs(z - np.floor(z)) - 0.5) > tie)).sum())
    assert differ <= 5e-4 * got.size + 3, f"{differ} of {got.size} codes differ"


def codes(rng, m, cols):
    """int8 codes whose rows resemble their neighbours'."""
    x = rng.normal(0, 28, (m, cols)) + np.repeat(rng.normal(0, 16, (m // 48 + 1, cols)), 48, axis=0)[:m]
    return np.clip(np.rint(x), -127, 127).astype(np.int8)


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
