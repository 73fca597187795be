"""GPU tests of attention_run against its definition in 64 bits with the bars of
attention_bars.py, the same for fp32 results and int8 codes."""
import numpy as np
import pytest

import attention_bars as bars

pytestmark = pytest.mark.gpu
T = 1  # LAYOUT_T16X32


def check(hip, x, lens, nh, nkv, hd, kind, xl=0, yl=0, x_scale=0.04, sm=None, key_len=None, lists=None, qb=64,
          max_len=None, step=bars.STEP, path=None):
    import torch
    m, start = len(x), bars.starts(lens)
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    xs = float(np.float32(x_scale))
    scale = float(np.float32(hd ** -0.5 if sm is None else sm))
    want, bar = bars.attention(x, xs, start, nh, nkv, hd, scale, key_len, lists, qb, step)
    so = bars.output_scale(want)
    longest = max(lens) if max_len is None else max_len
    print(f"attention {list(lens)[:8]} heads={nh}/{nkv}x{hd} kind={kind} layouts=({xl},{yl}) qb={qb}", flush=True)
    xd = torch.from_numpy(np.ascontiguousarray(hip.to_t16x32(x, fill=77) if xl == T else x)).cuda()
    y = hip.attention(xd, xs, dev(start), longest, nh, hd, n_kv_heads=nkv, softmax_scale=sm, key_len=dev(key_len),
                      kind=kind, out_scale=so, blocks=dev(lists), query_block=qb, x_layout=xl, y_layout=yl, m_tokens=m)
    torch.cuda.synchronize()
    if path is not None:
        assert hip.last_path() == "attention " + path
    got = y.cpu().numpy()
    got = hip.from_t16x32(got, m, nh * hd) if yl == T else got
    used = start[-1]
    bars.assert_within(got[:used], want[:used], bar[:used], so if kind == 3 else None)
    return got


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("hd", [16, 32, 48, 64, 80, 96, 112, 128])
def test_every_head_size(hip, hd, kind):
    rng = np.random.default_rng([hd, kind])
    lens = [128, 1, 65, 0, 200, 64, 385, 31]
    for nh, nkv, xl in ((4, 4, 0), (6, 2, T)):
        check(hip, bars.codes(rng, sum(lens), (nh + 2 * nkv) * hd), lens, nh, nkv, hd, kind, xl)


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("b,n,nh", [(32, 128, 4), (3, 384, 12), (1, 1000, 2), (1, 4097, 1), (40, 257, 4)])
def test_batches(hip, b, n, nh, kind):
    rng = np.random.default_rng([b, n])
    check(hip, bars.codes(rng, b * n, 3 * nh * 64), [n] * b, nh, nh, 64, kind, T, T if kind == 3 else 0)


@pytest.mark.parametrize("qb", [16, 32, 64, 128])
def test_lists(hip, qb):
    rng = np.random.default_rng(qb)
    lens, keys, nh = [700, 1, 64, 0, 333, 129], [700, 1, 0, 0, 300, 65], 3
    blocks = -(-700 // 64)
    lists = rng.permuted(np.tile(np.arange(blocks), (len(lens), nh, -(-700 // qb), 1)), axis=-1)[..., :5]
    for hd in (32, 64, 96, 128):
        x = bars.codes(rng, sum(lens), 3 * nh * hd)
        for kind in (1, 3):
            check(hip, x, lens, nh, nh, hd, kind, key_len=keys, lists=lists, qb=qb)


# lengths whose last 256, 32 and 64 tokens end everywhere, none shorter than nothing
MANY = [1030, 1, 257, 64, 1099, 0, 255, 1024, 31, 300, 65, 512]


@pytest.mark.parametrize("hd,padded", [(16, 32), (32, 32), (48, 64), (64, 64)])
@pytest.mark.parametrize("nh,nkv,kind,xl,yl,masked", [(12, 12, 1, 0, 0, False), (12, 3, 3, T, T, True),
                                                      (12, 12, 3, 0, T, True), (12, 4, 1, T, 0, True)])
def test_two_tiles_a_wave(hip, hd, padded, nh, nkv, kind, xl, yl, masked):
    """Many sequences of 1024 tokens and more, and of every other length among them."""
    rng = np.random.default_rng([hd, nh, nkv, kind])
    keys = [1030, 0, 200, 63, 1, 0, 255, 960, 17, 299, 64, 450] if masked else None
    x = bars.codes(rng, sum(MANY) + 3, (nh + 2 * nkv) * hd)  # (the last tokens belong to no sequence)
    check(hip, x, MANY, nh, nkv, hd, kind, xl, yl, key_len=keys, path=f"{padded},2,4,1")


@pytest.mark.parametrize("hd,padded", [(32, 32), (64, 64)])
def test_two_tiles_a_wave_where_scores_grow(hip, hd, padded):
    """m moves again and again, in the short last chunk too."""
    rng = np.random.default_rng(hd)
    nh = 12
    x = bars.codes(rng, sum(MANY), 3 * nh * hd)
    grow = np.concatenate([np.linspace(0.02, 1.0, n) for n in MANY])[:, None]
    cols = slice(nh * hd, 2 * nh * hd)
    x[:, cols] = np.clip(np.rint(x[:, cols] * grow * 2), -127, 127).astype(np.int8)
    for kind in (1, 3):
        check(hip, x, MANY, nh, nh, hd, kind, x_scale=0.15, path=f"{padded},2,4,1")


@pytest.mark.parametrize("lens,nh,hd,lists,path", [
    ([40] * 3, 2, 64, 0, "64,1,4,1"), ([300], 2, 64, 0, "64,1,1,4"), ([300], 2, 128, 0, "128,1,1,4"),
    ([1030] * 3, 8, 32, 0, "32,1,1,4"), ([300] * 30, 3, 96, 0, "96,1,4,1"), ([300] * 40, 4, 80, 0, "96,1,4,1"),
    ([300], 2, 64, 64, "64,1,1,4 lists"), ([300] * 30, 4, 64, 16, "64,1,1,1 lists"),
    ([300] * 30, 4, 64, 64, "64,1,2,1 lists"), ([300] * 30, 4, 64, 128, "64,1,4,1 lists"),
    ([300] * 30, 4, 128, 32, "128,1,4,1 lists")])
def test_other_shapes(hip, lens, nh, hd, lists, path):
    rng = np.random.default_rng([len(lens), nh, hd])
    x = bars.codes(rng, sum(lens), 3 * nh * hd)
    rows = None
    if lists:
        rows = rng.permuted(np.tile(np.arange(6), (len(lens), nh, -(-max(lens) // lists), 1)), axis=-1)[..., :4]
    for kind in (1, 3):
        check(hip, x, lens, nh, nh, hd, kind, lists=rows, qb=lists or 64, path=path)


def check_one_row(hip, n, hd, x, x_scale, sm, kind, step):
    """A sequence whose queries are all alike: its one row of results."""
    import torch
    xs, scale = float(np.float32(x_scale)), float(np.float32(sm))
    one = np.zeros((n, 3 * hd), np.int8)
    one[:1, :hd] = x[:1, :hd]
    one[:, hd:] = x[:, hd:]
    q, k, v = one[0, :hd].astype(np.float64), one[:, hd:2 * hd].astype(np.float64), one[:, 2 * hd:] * xs
    z = k @ q * (xs * xs * scale * np.log2(np.e))
    w = np.exp2(z - z.max())
    a = w @ np.abs(v) / w.sum()
    rel = 2.0 ** -23 + (z.max() - z.min() + 16) * 2.0 ** -22 + 2.0 ** -21
    bar = (2 * rel + (n / 4 + n / 64 + 32) * 2.0 ** -24) * a + step * np.abs(v).sum(0) / w.sum()
    want = w @ v / w.sum()
    so = bars.output_scale(want)
    y = hip.attention(torch.from_numpy(x).cuda(), xs, torch.tensor([0, n], dtype=torch.int32, device="cuda"), n, 1, hd,
                      softmax_scale=sm, kind=kind, out_scale=so).cpu().numpy()
    for got in (y[0], y[n // 2], y[-1]):
        bars.assert_within(got, want, bar, so if kind == 3 else None)
    assert (y == y[0]).all()


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("n,hd", [(500, 64), (20000, 64), (20000, 32), (3000, 128)])
def test_many_small_weights(hip, n, hd, kind):
    """Keys of 2^-14 to 2^-18 of one key's weight, which has no value: the results are theirs alone."""
    rng = np.random.default_rng([n, hd])
    x = np.zeros((n, 3 * hd), np.int8)
    x[:, 0], x[0, hd] = 100, 90
    x[1:, hd] = rng.integers(0, 20, n - 1)
    x[1:, 2 * hd:] = rng.integers(20, 120, (n - 1, hd))
    check_one_row(hip, n, hd, x, 0.1, 18 / (9000 * 0.01 * np.log2(np.e)), kind, bars.STEP)


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("octaves", [0.5, 1.3, 1.34, 1.41, 1.9, 2.6, 2.7, 3.3, 4.9, 5.4, 6.1, 9.7, 10.6, 10.7, 14.3, 40.0])
def test_small_weights_of_coarse_scores(hip, octaves, kind):
    """Scales at which a step of the whole-number scores is worth that many octaves of weight."""
    n, hd = 500, 64
    rng = np.random.default_rng(5)
    step = bars.STEP if octaves < 4 / 3 else 2.0 ** -28 if octaves < 32 / 3 else 2.0 ** -24
    for far in (9.0, 10.5, 12.0, 13.5):
        x = np.zeros((n, 3 * hd), np.int8)
        x[:, 0], x[0, hd] = 1, max(1, round(far / octaves))
        x[1:, 2 * hd:] = rng.integers(20, 120, (n - 1, hd))
        check_one_row(hip, n, hd, x, 1.0, octaves / np.log2(np.e), kind, step)
