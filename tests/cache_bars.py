"""How far results of cache_attention may be from their definition in 64 bits, and the definition with what these bars
need. Shares no code with the library.

For a query, with x_j <= 0 the exponents of the weights w_j = 2^x_j relative to the largest, n the keys that take part,
v_j codes of values, W = sum_j w_j, A = sum_j w_j |v_j| / W for every feature, and r = 2^-24, a rounding in 32 bits:

* An error d of every weight moves their mean by 2 d A, one that varies with j by sum_j d_j w_j (|v_j| + A) / W.
* Few queries ("split"; a wave takes every 4th span of 64 keys, so ceil(n / 256) of them, S):
  - The exponent's factor is rounded, and its product with a difference of scores, itself exact: 2 r |x_j| ln 2 of a
    weight. The product is taken in pieces of one sign (to the span's largest score, the wave's, the workgroup's, the
    parts'), whose roundings together are no more. Every piece has an exponential, off by 2 r: those four, and one for
    each span of a wave at which its largest score moves.
  - A weight is a whole number of 8355000ths of its span's largest, T_j: an absolute error of 0.5 / 8355000 of that, in the
    sum of weights too: sum_j T_j (|v_j| + A) / W of it. (Spans begin at slots that are multiples of 64.)
  - Sums of a span are exact; the conversion of the lower two digits' sum and the sum of all three round (2 r). A span
    joins a wave's by two products and a sum (3 r), four waves meet by a product each and three sums, p parts by a
    product each and p sums, and a division and two products end it: 3 S + p + 16 in the numerator, and in W.
* Many queries ("prompt"; chunks of 64 keys, ceil(n / 64) of them, C):
  - The factor is held in 22 bits, and its product with a score, to which up to 8 is added, rounds once: (3 |x_j| + 8) r
    ln 2 of a weight, the exponential 2 r. One more exponential for each chunk at which the largest score moves, and for waves' and parts'.
  - The first 16-bit part is the weight cut to 11 bits, the second what that leaves, cut to 11 bits: 2^-20 of the weight,
    which the sum of weights does not share. 16-bit floats end at a step of 2^-24, and weights carry a factor of 2^7:
    an absolute error of up to 2^-31 of the largest.
  - Products are added in fp32, four for a chunk's 16 keys each and two parts (n / 4 roundings in all of two a product);
    the sum of weights n / 64 + 32, and a rescaling of each for a chunk.
"""
import numpy as np

import cache_ref as ref

R = 2.0 ** -24
LN2 = float(np.log(2.0))


def attention(q, cache, start, lens, table, nh, scale, causal, form, parts=1, weights=lambda w: w):
    """y [M, nh * hd] in codes of values, as float64, their bars, and which tokens have a sequence. `weights`: applied to
    the weights that meet v (and, of few queries, to those summed)."""
    n_pages, _, nkv, ps, hd = cache.shape
    m, g = len(q), nh // nkv
    y, bar, real = np.zeros((m, nh, hd)), np.zeros((m, nh, hd)), np.zeros(m, bool)
    groups = cache[:, 1].reshape(n_pages, nkv, ps // 16, hd, 16)
    for s in range(len(lens)):
        first, end, length = int(start[s]), int(start[s + 1]), max(int(lens[s]), 0)
        real[first:end] = True
        where = [(i, page, place) for i, (page, place) in enumerate(ref.slots_of(table, ps, n_pages, s, length)) if page >= 0]
        if first == end or not where:
            continue
        at, page, place = np.array(where, dtype=np.int64).T
        last = length - (end - first) + np.arange(end - first) if causal else np.full(end - first, length - 1)
        seen = np.repeat(at[None] <= last[:, None], g, 0)  # [tokens * group, keys]
        some, n = seen.any(1)[:, None], seen.sum(1)[:, None]
        for h in range(nkv):
            k = cache[page, 0, h, place].astype(np.float64)
            v = groups[page, h, place // 16, :, place % 16].astype(np.float64)
            rows = q[first:end, h * g * hd:(h + 1) * g * hd].reshape(-1, hd).astype(np.float64)
            x = np.where(seen, rows @ k.T * (scale * np.log2(np.e)), -np.inf)
            x = np.where(seen, x - np.where(some, x.max(1, keepdims=True), 0.0), -np.inf)
            w = np.exp2(x)
            far = np.where(seen, -x, 0.0) * w
            total = np.where(some, w.sum(1, keepdims=True), 1.0)
            mag = np.abs(v)
            a = w @ mag / total
            varied = (far @ mag + far.sum(1, keepdims=True) * a) / total
            first_of = np.flatnonzero(np.diff(at // 64, prepend=-1))  # (slots ascend)
            tops = np.maximum.reduceat(w, first_of, axis=1)  # of spans
            tops = np.where(seen, np.repeat(tops, np.diff(np.append(first_of, len(at))), 1), 0.0)
            whole = (tops @ mag + tops.sum(1, keepdims=True) * a) / total
            met = np.where(seen, weights(w), 0.0)
            if form == "split":
                summed, spans = met, np.ceil(n / 256)
                d = 2 * R * LN2 * varied + 2 * (4 + spans) * 2 * R * a + whole * 0.5 / 8355000 * (1 + 2.0 ** -10)
                rounded = 2 * (3 * spans + parts + 16) * R
            else:
                summed, chunks = w, np.ceil(n / 64)
                d = 3 * R * LN2 * varied + 2 * (8 * LN2 * R + (3 + chunks) * 2 * R) * a + 2.0 ** -20 * a
                d += 2.0 ** -31 * (seen @ mag) / total
                rounded = (n / 4 + n / 64 + 32 + 2 * chunks + 2 * parts + 8) * R
            out = met @ v / np.where(some, summed.sum(1, keepdims=True), 1.0)
            y[first:end, h * g:(h + 1) * g] = out.reshape(-1, g, hd)
            bar[first:end, h * g:(h + 1) * g] = np.where(some, d + rounded * a, 0.0).reshape(-1, g, hd)
    return y.reshape(m, -1), bar.reshape(m, -1), real
