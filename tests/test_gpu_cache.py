"""cache_append and cache_attention on the GPU against the 64-bit definitions of cache_ref.py.

Bars.
- Stored codes and query codes: within half a step and DELTA of value / scale. The angle is rounded to 2^-25 turns
  (1.9e-7 radians), its sine and cosine to a few 2^-24: together under 6e-7; a rotated value is two products and a sum of
  them (3 more roundings of 2^-24), and the factor to codes one more: under 1.2e-6 of |a| + |b|, which with |a|, |b| <=
  127 * 1.2 steps is 4e-4 steps. DELTA = 1e-3.
- Attention: the weights' relative error is that of the exponential's argument x <= 24 that matters, |x| 2^-23 ln 2 (its
  factor's and its product's rounding), weighted with 2^-x under 1e-7 of the largest, over many keys of which each
  weighs little at most 24 * 2^-23 * ln 2 = 2e-6; the instruction's own 2^-22; and the whole number that stands for a
  weight, 2^-24 of its span's largest, which the up to 128 keys of a span, all rounded one way, could add up to 2^-17
  (the sum of weights moves with it). Sums in 32 bits: 2^-24 for each of up to 100 additions, 6e-6. Together under 2e-5
  of the largest |v| = 127 v_scale, for the numerator and again for the denominator: TOL = 4e-5 * 127 v_scale.
"""
import numpy as np
import pytest

import cache_ref as ref

pytestmark = pytest.mark.gpu

DELTA = 1e-3
TOL = 4e-5 * 127
FILL = -77  # what outputs hold before a call


def codes(rng, *shape):
    return np.clip(np.rint(rng.standard_normal(shape) * 32), -127, 127).astype(np.int8)


class Batch:
    """Sequences with news[i] tokens of the call and lens[i] cached ones, their pages in any order."""

    def __init__(self, hip, rng, news, lens, ps, nkv, hd, spare=3, gap=0, holes=False):
        import torch
        self.hip, self.news, self.lens, self.nkv, self.hd, self.ps = hip, news, lens, nkv, hd, ps
        self.start = np.concatenate([[gap], gap + np.cumsum(news)]).astype(np.int32)
        self.m = int(self.start[-1]) + gap  # (gap tokens of no sequence at either end)
        self.len = np.array(lens, np.int32)
        count = [max(0, -(-n // ps)) for n in lens]
        per = max(count + [0]) + 1
        self.n_pages = sum(count) + spare
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.table = np.full((len(news), per), -1, np.int32)
        at = 0
        for s, c in enumerate(count):
            self.table[s, :c] = order[at:at + c]
            at += c
        if holes:  # pages that are none in the middle of a sequence
            self.table[rng.random(self.table.shape) < 0.25] = -1
            self.table[0, 0] = self.n_pages
        self.cache = codes(rng, *hip.cache_shape(self.n_pages, ps, nkv, hd))
        c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        self.dev = [c(a) for a in (self.cache, self.table, self.start, self.len)]
        self.most_new, self.longest = max(news), max(max(lens), 0)


def filled(hip, shape, dtype):
    import torch
    return torch.full(shape, FILL, dtype=dtype, device="cuda")


def run_append(hip, rng, b, nh, x_type="i8", kind=ref.HALF, rot=None, factor=1.0, layout=0, positions=None, scales=None):
    import torch
    hd, nkv = b.hd, b.nkv
    rot = hd if rot is None else rot
    cols = (nh + 2 * nkv) * hd
    xs, qs, ks, vs = scales or (0.031, 0.037, 0.041, 0.031)
    f = np.float32
    if x_type == "i8":
        x = codes(rng, b.m, cols)
        value = x.astype(np.float64) * float(f(xs))
        dev = torch.from_numpy(hip.to_t16x32(x) if layout else x).cuda()
    else:
        x = rng.standard_normal((b.m, cols)).astype(f)
        value, xs = x.astype(np.float64), 1.0
        dev = torch.from_numpy(x).cuda()
    freq = (10000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))).astype(f)
    cache, table, start, lens = b.dev
    out = filled(hip, hip.t16x32_shape(b.m, nh * hd) if layout else (b.m, nh * hd), torch.int8) if nh else None
    q = hip.cache_append(dev, cache, table, start, lens, b.most_new, nh, x_scale=xs, q_scale=qs if nh else None, k_scale=ks,
                         v_scale=vs, rope=kind, inv_freq=torch.from_numpy(freq).cuda() if kind else None,
                         rope_factor=factor, positions=None if positions is None else torch.from_numpy(positions).cuda(),
                         x_layout=layout, q_layout=layout, m_tokens=b.m, out=out)
    torch.cuda.synchronize()
    factor = float(f(factor))
    queries, stored = ref.append(value, b.start, b.len, b.table, b.ps, b.n_pages, nh, nkv, hd, kind, freq, factor, positions)
    want = b.cache.copy()
    got = cache.cpu().numpy()

    def near(code, v, scale):
        v = np.clip(v / float(f(scale)), -127, 127)
        assert np.abs(code.astype(np.float64) - v).max() <= 0.5 + DELTA

    for page, place, k, v in stored:
        for h in range(nkv):
            near(ref.key_of(got, page, h, place), k[h], ks)
            near(ref.value_of(got, page, h, place), v[h], vs)
            ref.key_of(want, page, h, place)[:] = ref.key_of(got, page, h, place)
            ref.value_of(want, page, h, place)[:] = ref.value_of(got, page, h, place)
    assert np.array_equal(got, want), "bytes of other slots changed"
    if nh:
        assert q is out
        rows = hip.from_t16x32(q.cpu().numpy(), b.m, nh * hd) if layout else q.cpu().numpy()
        for t in range(b.m):
            if t in queries:
                near(rows[t].reshape(nh, hd), queries[t], qs)
            else:
                assert (rows[t] == FILL).all()
    else:
        assert q is None
    return value, got


@pytest.mark.parametrize("news,lens", [([1], [1]), ([1], [100]), ([1, 1, 1], [16, 17, 0]), ([5, 1, 40, 3], [5, 33, 47, 3]),
                                       ([4, 19], [2, 300])])
@pytest.mark.parametrize("x_type,layout", [("i8", 0), ("i8", 1), ("f32", 0)])
@pytest.mark.parametrize("kind", [ref.NONE, ref.HALF, ref.INTERLEAVED])
def test_append(hip, news, lens, x_type, layout, kind):
    rng = np.random.default_rng(len(news) * 100 + news[0])
    b = Batch(hip, rng, news, lens, 16, 2, 64, gap=3)
    run_append(hip, rng, b, 4, x_type, kind, layout=layout)


@pytest.mark.parametrize("hd,rot,ps,nh,nkv", [(16, 16, 32, 3, 3), (16, 2, 16, 1, 1), (48, 18, 64, 8, 2), (80, 80, 128, 5, 1),
                                              (96, 24, 256, 2, 2), (128, 126, 16, 4, 4), (128, 64, 32, 16, 2)])
@pytest.mark.parametrize("kind", [ref.HALF, ref.INTERLEAVED])
@pytest.mark.parametrize("x_type", ["i8", "f32"])
def test_append_heads_and_pages(hip, hd, rot, ps, nh, nkv, kind, x_type):
    rng = np.random.default_rng(hd + rot)
    b = Batch(hip, rng, [7, 1, 18], [9, 50, 18], ps, nkv, hd)
    run_append(hip, rng, b, nh, x_type, kind, rot)


def test_append_keys_and_values_only(hip):
    rng = np.random.default_rng(5)
    run_append(hip, rng, Batch(hip, rng, [40, 3], [40, 3], 16, 3, 32), 0, "i8", ref.NONE)


def test_append_far_positions_and_factor(hip):
    rng = np.random.default_rng(6)
    b = Batch(hip, rng, [6, 2], [9, 2], 16, 2, 64)
    pos = np.array([0, 1, 131071, 1048575, 2 ** 31 - 1, -5, 77777, 3], np.int32)
    run_append(hip, rng, b, 2, "f32", ref.HALF, factor=1.13, positions=pos, scales=(1.0, 0.05, 0.05, 0.05))


def test_append_leaves_out_what_has_no_page(hip):
    rng = np.random.default_rng(7)
    b = Batch(hip, rng, [60, 9, 4], [90, 9, 2], 16, 2, 32, holes=True)
    run_append(hip, rng, b, 2)
    b = Batch(hip, rng, [3, 2], [40, 20], 16, 2, 32)
    b.table = np.ascontiguousarray(b.table[:, :1])  # slots behind the table
    import torch
    b.dev[1] = torch.from_numpy(b.table).cuda()
    run_append(hip, rng, b, 2)


def test_append_more_tokens_than_said(hip):
    rng = np.random.default_rng(8)
    b = Batch(hip, rng, [21, 2], [30, 2], 16, 1, 16)
    b.most_new = 1
    run_append(hip, rng, b, 1)


def test_equal_scales_copy_codes(hip):
    rng = np.random.default_rng(9)
    b = Batch(hip, rng, [33], [40], 16, 2, 64)
    value, got = run_append(hip, rng, b, 2, "i8", ref.NONE, scales=(0.031,) * 4)
    page, place = ref.slots_of(b.table, 16, b.n_pages, 0, 40)[12]
    x = np.rint(value[5].reshape(6, 64) / np.float32(0.031))
    assert np.array_equal(ref.key_of(got, page, 1, place), x[3]) and np.array_equal(ref.value_of(got, page, 0, place), x[4])


def run_attend(hip, rng, b, nh, kind="f32", causal=True, q_layout=0, y_layout=0, wide=0, qs=0.04, ks=0.05, scale=None,
               q=None, stream=None):
    import torch
    hd, vs, f = b.hd, 0.03, np.float32
    q = codes(rng, b.m, nh * hd + wide) if q is None else q
    cache, table, start, lens = b.dev
    scale = hd ** -0.5 if scale is None else scale
    want, _ = ref.attention(q, b.cache, b.start, b.len, b.table, nh, float(f(qs)) * float(f(ks)) * float(f(scale)), causal)
    so = max([float(np.abs(v).max()) for v in want.values()] + [1e-3]) * vs / 120
    i8 = kind == "i8"
    out = filled(hip, hip.t16x32_shape(b.m, nh * hd) if y_layout else (b.m, nh * hd), torch.int8 if i8 else torch.float32)
    y = hip.cache_attention(torch.from_numpy(hip.to_t16x32(q) if q_layout else q).cuda(), cache, table, start, lens,
                            b.most_new, b.longest, nh, q_scale=qs, k_scale=ks, v_scale=vs, softmax_scale=scale,
                            causal=causal, kind=hip.EPI_I8 if i8 else hip.EPI_F32, out_scale=so, q_layout=q_layout,
                            q_cols=nh * hd + wide, y_layout=y_layout, m_tokens=b.m, out=out, stream=stream)
    torch.cuda.synchronize()
    assert y is out
    rows = hip.from_t16x32(y.cpu().numpy(), b.m, nh * hd) if y_layout else y.cpu().numpy()
    worst = 0.0
    for t in range(b.m):
        if t not in want:
            assert (rows[t] == FILL).all()
            continue
        v = want[t].reshape(-1) * float(f(vs))
        if i8:
            off = np.abs(rows[t] - np.clip(v / float(f(so)), -127, 127)).max() - 0.5
            assert off <= TOL * vs / so + 1e-3, (t, off)
        else:
            worst = max(worst, float(np.abs(rows[t] - v).max()) / (127 * vs))
            assert np.isfinite(rows[t]).all() and worst <= TOL / 127, (t, worst)
    return rows


CASES = [([1], [1]), ([1], [15]), ([1], [64]), ([1], [129]), ([1], [2000]), ([1, 1, 1, 1], [700, 0, 1, 513]),
         ([3, 1, 5], [300, 260, 5]), ([40, 1, 17], [40, 33, 90]), ([200], [200]), ([130, 2], [1000, 7]), ([9, 6], [4, 2])]


@pytest.mark.parametrize("news,lens", CASES)
@pytest.mark.parametrize("nh,nkv,hd", [(2, 2, 64), (8, 2, 128), (6, 1, 48)])
@pytest.mark.parametrize("causal", [True, False])
def test_attention(hip, news, lens, nh, nkv, hd, causal):
    rng = np.random.default_rng(news[0] * 7 + hd)
    run_attend(hip, rng, Batch(hip, rng, news, lens, 16, nkv, hd, gap=2), nh, causal=causal)


@pytest.mark.parametrize("hd", range(16, 129, 16))
@pytest.mark.parametrize("ps", [16, 32, 64, 128, 256])
def test_attention_heads_and_pages(hip, hd, ps):
    rng = np.random.default_rng(hd + ps)
    run_attend(hip, rng, Batch(hip, rng, [1, 2, 1, 33], [700, 300, 17, 130], ps, 2, hd), 6)


@pytest.mark.parametrize("news,lens", [([1, 1], [900, 40]), ([70, 9], [400, 9])])
@pytest.mark.parametrize("q_layout,y_layout,wide", [(0, 0, 0), (0, 0, 64), (1, 0, 0), (1, 1, 16), (0, 1, 16)])
def test_attention_layouts(hip, news, lens, q_layout, y_layout, wide):
    rng = np.random.default_rng(11)
    b = Batch(hip, rng, news, lens, 32, 2, 64, gap=5)
    run_attend(hip, rng, b, 4, "i8", q_layout=q_layout, y_layout=y_layout, wide=wide)


@pytest.mark.parametrize("news,lens", [([1, 1, 1], [900, 40, 300]), ([70, 9], [400, 90])])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_pages_that_are_none(hip, news, lens, causal):
    rng = np.random.default_rng(12)
    run_attend(hip, rng, Batch(hip, rng, news, lens, 16, 2, 64, holes=True), 4, causal=causal)


def test_attention_without_pages(hip):
    import torch
    rng = np.random.default_rng(13)
    b = Batch(hip, rng, [2, 30], [5, 40], 16, 1, 32)
    b.table[:] = -1
    b.dev[1] = torch.from_numpy(b.table).cuda()
    assert (run_attend(hip, rng, b, 2) == 0).all()
    b.table = b.table[:, :0]
    b.dev[1] = torch.from_numpy(np.ascontiguousarray(b.table)).cuda()
    assert (run_attend(hip, rng, b, 2) == 0).all()
    b.cache = b.cache[:0]
    b.dev[0] = b.dev[0][:0]
    b.n_pages = 0
    assert (run_attend(hip, rng, b, 2) == 0).all()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("qs,ks", [(1e-20, 1e-20), (1e-4, 1e-3), (3.0, 2.0), (1e6, 1e6)])
def test_attention_scales(hip, new, qs, ks):
    """Flat weights, and rows where one key has all of it."""
    rng = np.random.default_rng(14)
    run_attend(hip, rng, Batch(hip, rng, [new], [600], 16, 2, 64), 4, qs=qs, ks=ks)


@pytest.mark.parametrize("new", [1, 33])
def test_attention_largest_codes(hip, new):
    """Scores at both ends of what the integers hold, a code of -128 among them."""
    import torch
    rng = np.random.default_rng(15)
    b = Batch(hip, rng, [new], [500], 16, 1, 128)
    b.cache[:] = rng.choice(np.array([-128, 127], np.int8), b.cache.shape)
    b.dev[0] = torch.from_numpy(b.cache).cuda()
    q = np.sign(rng.standard_normal((b.m, 256))).astype(np.int8) * 127
    q[:, :128] = b.cache[b.table[0, 3], 0, 0, 5] // 2 * 2 + (b.cache[b.table[0, 3], 0, 0, 5] > 0)
    run_attend(hip, rng, b, 2, q=np.ascontiguousarray(np.maximum(q, -127)), qs=0.002, ks=0.05)


@pytest.mark.parametrize("new", [1, 50])
def test_attention_more_than_said(hip, new):
    """More new tokens and longer sequences than the launch is sized by."""
    rng = np.random.default_rng(16)
    b = Batch(hip, rng, [new + 3, new, new + 40], [3000, 700, 1500], 16, 2, 64)
    b.most_new, b.longest = new, 1000
    run_attend(hip, rng, b, 4)
    b.longest = 0
    run_attend(hip, rng, b, 4)


@pytest.mark.parametrize("nh,nkv", [(16, 1), (17, 1), (40, 2), (100, 1)])
@pytest.mark.parametrize("news,lens", [([1, 1], [600, 33]), ([3, 20], [30, 700])])
def test_attention_large_groups(hip, nh, nkv, news, lens):
    """More query heads a key head than a tile has rows."""
    rng = np.random.default_rng(nh)
    run_attend(hip, rng, Batch(hip, rng, news, lens, 32, nkv, 32), nh)


def test_attention_many_sequences(hip):
    rng = np.random.default_rng(17)
    lens = [int(n) for n in rng.integers(0, 90, 700)]
    run_attend(hip, rng, Batch(hip, rng, [1] * 700, lens, 16, 1, 16), 1)


@pytest.mark.parametrize("news,lens", [([40], [5000]), ([130, 3, 1], [3000, 2050, 1]), ([33, 129], [2049, 140])])
@pytest.mark.parametrize("nh,nkv,hd", [(2, 2, 64), (4, 1, 128), (3, 1, 16)])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_many_queries_in_parts(hip, news, lens, nh, nkv, hd, causal):
    rng = np.random.default_rng(news[0] + hd)
    run_attend(hip, rng, Batch(hip, rng, news, lens, 16, nkv, hd, gap=1, holes=hd == 16), nh, causal=causal)


@pytest.mark.parametrize("new", [2, 50])
def test_attention_in_parts_of_more_than_said(hip, new):
    rng = np.random.default_rng(19)
    b = Batch(hip, rng, [new + 30, new, 140], [6000, 700, 2500], 16, 1, 64)
    b.most_new, b.longest = new, 2100
    run_attend(hip, rng, b, 2)


# prompts of different lengths, more than a workgroup for every CU: tiles in order of the keys that they see
SORTED = [([100, 0, 7, 64, 65, 130, 1, 33], [100, 50, 300, 64, 1000, 140, 0, 33]), ([128, 128, 3, 128, 60], [128, 700, 3, 700, 2]),
          ([300, 40], [300, 2300]), ([40] + [5, 0, 1] * 21, [41] + [70, 0, 9] * 21)]


@pytest.mark.parametrize("news,lens", SORTED)
@pytest.mark.parametrize("nh,nkv,hd", [(40, 40, 16), (24, 24, 64), (60, 20, 96), (24, 24, 128), (200, 2, 32)])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_in_order_of_length(hip, news, lens, nh, nkv, hd, causal):
    rng = np.random.default_rng(20)
    run_attend(hip, rng, Batch(hip, rng, news, lens, 16, nkv, hd, gap=1, holes=hd == 64), nh, causal=causal)


@pytest.mark.parametrize("longest", [100, 2100])  # (the second in two parts)
def test_attention_in_order_of_more_than_said(hip, longest):
    rng = np.random.default_rng(21)
    b = Batch(hip, rng, [3, 140] + [5] * 20, [30, 2600] + [90] * 20, 16, 20, 64)
    b.most_new, b.longest = 30, longest
    run_attend(hip, rng, b, 20)
    assert hip.last_path() == f"cache prompt 64,{1 if longest == 100 else 2}"


@pytest.mark.parametrize("n,nh,nkv,hd", [(3, 4, 2, 64), (64, 8, 8, 16), (70, 16, 8, 128), (256, 3, 1, 96), (257, 2, 2, 32)])
@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_steps_that_may_be_long(hip, n, nh, nkv, hd, equal, causal):
    """Steps sized for 2^28 bytes of cache and more, where the sequences with the most keys come first."""
    rng = np.random.default_rng(n + hd)
    lens = [130] * n if equal else [int(k) for k in rng.integers(0, 300, n)]
    news = [1] * n if equal else [int(k) for k in rng.integers(0, 4, n)]
    b = Batch(hip, rng, news, lens, 16, nkv, hd, gap=2, holes=hd == 16)
    b.longest = 2 ** 28 // (n * nkv * 2 * hd) + 1
    run_attend(hip, rng, b, nh, causal=causal)
    b.most_new = 1  # (where some have more)
    run_attend(hip, rng, b, nh, causal=causal)


def test_attention_of_long_steps_in_parts(hip):
    rng = np.random.default_rng(22)
    b = Batch(hip, rng, [1, 3, 1, 0, 1, 1], [5000, 40, 9000, 700, 0, 2600], 64, 2, 128)
    b.longest = 90000
    run_attend(hip, rng, b, 8)
    assert hip.last_path() == "cache split 128,40"  # of 90000 / 43 keys, up to the next 256: 2304


def test_attention_long(hip):
    rng = np.random.default_rng(18)
    run_attend(hip, rng, Batch(hip, rng, [1, 2], [40000, 9999], 64, 1, 64), 8)
