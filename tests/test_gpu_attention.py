"""GPU tests of attention and select_blocks through the C ABI against their
definitions in 64 bits.

Bars. A weight 2^e is off by a relative 2^-23 (the exponential), |e| 2^-23 (the
exponent's rounding) and |e| 2^-22 (the factor of the scores, held in 22 bits);
|e| <= 1.45 times the spread of a row's logits. Rounding it to the products' 16
bits (toward zero) takes up to 2^-10 for int8 results; fp32 results carry the
rest in a second product, which leaves 2^-20. A relative error d of the weights
moves a weighted mean by at most 2 d max|v|, since the sum of weights is taken
from the rounded ones. The fp32 sums over n keys add at most (n / 16) 2^-24
max|v|. Chosen blocks have to be equal.
"""
import numpy as np
import pytest

import encoder_ref as ref

pytestmark = pytest.mark.gpu
T = 1  # LAYOUT_T16X32


def _codes(rng, m, cols, low=-127):
    """Codes whose rows resemble their neighbours'."""
    x = rng.normal(0, 28, (m, cols)) + np.repeat(rng.normal(0, 16, (m // 48 + 1, cols)), 48, axis=0)[:m]
    return np.clip(np.rint(x), low, 127).astype(np.int8)


def _starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _dev(hip, x, layout):
    import torch
    return torch.from_numpy(np.ascontiguousarray(hip.to_t16x32(x, fill=77) if layout == T else x)).cuda()


def _check(hip, x, lens, nh, nkv, hd, kind, xl=0, yl=0, x_scale=0.04, sm=None, key_len=None, lists=None, qb=64,
           max_len=None, say=""):
    import torch
    m = len(x)
    start = _starts(lens)
    i32 = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    xs = float(np.float32(x_scale))
    scale = float(np.float32(hd ** -0.5 if sm is None else sm))
    want, spread = ref.attention(x, xs, start, nh, nkv, hd, scale, key_len, lists, qb)
    e = 1.45 * spread
    n = max(list(lens) + [1])
    vmax = 128 * xs
    rel = 2.0 ** -23 + e * (2.0 ** -23 + 2.0 ** -22) + (2.0 ** -10 if kind == 3 else 2.0 ** -20)
    bar = vmax * (2 * rel + (n / 16 + 8) * 2.0 ** -24)
    so = float(np.float32(max(np.abs(want).max(), 1e-3) / 126))
    print(f"attention {say} m={m} heads={nh}/{nkv}x{hd} kind={kind} layouts=({xl},{yl}) qb={qb}", flush=True)
    y = hip.attention(_dev(hip, x, xl), xs, i32(start), max(lens) if max_len is None else max_len, nh, hd,
                      n_kv_heads=nkv, softmax_scale=sm, key_len=i32(key_len), kind=kind, out_scale=so,
                      blocks=i32(lists), query_block=qb, x_layout=xl, y_layout=yl, m_tokens=m)
    torch.cuda.synchronize()
    got = y.cpu().numpy()
    used = start[-1]
    if kind == 1:
        off = np.abs(got[:used].astype(np.float64) - want[:used])
        assert np.isfinite(off).all() and (off.size == 0 or off.max() <= bar), f"{off.max()} against {bar}"
    else:
        got = hip.from_t16x32(got, m, nh * hd) if yl == T else got
        off = np.abs(got[:used] - np.clip(want[:used] / so, -127, 127))
        assert off.size == 0 or off.max() <= 0.5 + bar / so + 1e-4, f"{off.max()} against {0.5 + bar / so}"
    return got


LENS = [1, 2, 15, 16, 17, 63, 64, 65, 0, 127, 128, 129, 200, 385]


@pytest.mark.parametrize("hd", [16, 32, 48, 64, 80, 96, 112, 128])
@pytest.mark.parametrize("kind", [1, 3])
def test_head_sizes_and_lengths(hip, hd, kind):
    rng = np.random.default_rng(hd)
    for nh, nkv, xl, yl in [(2, 2, 0, 0), (3, 1, T, 0), (4, 2, T, T), (1, 1, 0, T)]:
        if yl == T and kind == 1:
            continue
        x = _codes(rng, sum(LENS), (nh + 2 * nkv) * hd)
        _check(hip, x, LENS, nh, nkv, hd, kind, xl, yl)


@pytest.mark.parametrize("n", [1, 5, 16, 31, 64, 100, 128, 384, 1000, 4097])
@pytest.mark.parametrize("kind", [1, 3])
def test_one_sequence(hip, n, kind):
    rng = np.random.default_rng(n)
    _check(hip, _codes(rng, n, 3 * 2 * 64), [n], 2, 2, 64, kind)


@pytest.mark.parametrize("b,n", [(32, 128), (3, 384), (150, 20), (400, 70)])
def test_batches(hip, b, n):
    rng = np.random.default_rng(b)
    for kind, xl, yl in ((3, T, T), (1, 0, 0)):
        _check(hip, _codes(rng, b * n, 3 * 4 * 64), [n] * b, 4, 4, 64, kind, xl, yl)


@pytest.mark.parametrize("kind", [1, 3])
def test_masked_keys(hip, kind):
    """Valid keys that end inside a tile, a block, at nothing; the queries past them are computed too."""
    rng = np.random.default_rng(9)
    lens = [100, 100, 100, 257, 257, 64, 1, 130]
    keys = [0, 1, 99, 64, 65, 63, 0, 130]
    x = _codes(rng, sum(lens), 3 * 2 * 64)
    got = _check(hip, x, lens, 2, 2, 64, kind, key_len=keys)
    assert not got[:100].any() and got[100:200].any()


def test_masked_values_do_not_matter(hip):
    """Keys and values beyond key_len, tokens of no sequence and padding of the block layout reach no result."""
    import torch
    rng = np.random.default_rng(2)
    lens, keys = [90, 70], [50, 64]
    x = _codes(rng, 160 + 9, 3 * 64)
    other = x.copy()
    other[50:90, 64:], other[90 + 64:160, 64:], other[160:] = 127, -127, -128
    for xl in (0, T):
        a = _check(hip, x, lens, 1, 1, 64, 1, xl, key_len=keys)
        b = _check(hip, other, lens, 1, 1, 64, 1, xl, key_len=keys)
        assert np.array_equal(a[:160], b[:160])


@pytest.mark.parametrize("x_scale,sm", [(1e-4, None), (0.02, None), (0.3, None), (1.0, 1.0), (3.0, 10.0), (1.0, 1e-9)])
@pytest.mark.parametrize("kind", [1, 3])
def test_sharp_and_flat_softmax(hip, x_scale, sm, kind):
    """From uniform weights to a single key with weight one; the running maximum grows late."""
    rng = np.random.default_rng(5)
    for hd in (64, 128):
        x = _codes(rng, 300, 3 * hd)
        x[:, hd:2 * hd] = np.clip(x[:, hd:2 * hd] * np.linspace(0.05, 1.0, 300)[:, None], -127, 127).astype(np.int8)
        _check(hip, x, [300], 1, 1, hd, kind, x_scale=x_scale, sm=sm)


def test_largest_scores(hip):
    """Scores of either sign at the end of their range, -128 among the codes, in one row."""
    for hd in (64, 128):
        for qv in (-128, 127):
            x = np.full((200, 3 * hd), 3, np.int8)
            x[:, :hd] = qv
            x[0::2, hd:2 * hd], x[1::2, hd:2 * hd] = -128, 127
            x[:, 2 * hd:] = np.arange(200)[:, None] - 100
            for kind in (1, 3):
                _check(hip, x, [200], 1, 1, hd, kind, x_scale=0.01)
                _check(hip, x, [200], 1, 1, hd, kind, x_scale=1.0, sm=1.0)


def test_one_key_among_many_small_ones(hip):
    """A key of large weight and thousands whose weights are each far below it but make up half of the sum."""
    n, hd = 6000, 64
    x = np.zeros((n, 3 * hd), np.int8)
    x[:, 0], x[0, hd], x[:, 2 * hd:] = 100, 87, 50
    x[0, 2 * hd:] = -100
    for kind in (1, 3):
        _check(hip, x, [n], 1, 1, hd, kind, x_scale=0.1, sm=0.1)  # weight of key 0: e^8.7 = 6003


def test_max_len_may_be_short_or_long(hip):
    rng = np.random.default_rng(8)
    x = _codes(rng, 500, 3 * 64)
    for max_len in (1, 100, 5000):
        _check(hip, x, [300, 200], 1, 1, 64, 1, max_len=max_len)


def test_starts_outside_the_tokens_are_brought_in(hip):
    import torch
    x = torch.from_numpy(_codes(np.random.default_rng(1), 64, 3 * 64)).cuda()
    start = torch.tensor([-5, 40, 30, 1000], dtype=torch.int32, device="cuda")
    y = hip.attention(x, 0.04, start, 64, 1, 64, kind=1)
    want = hip.attention(x, 0.04, torch.tensor([0, 40, 64], dtype=torch.int32, device="cuda"), 64, 1, 64, kind=1)
    torch.cuda.synchronize()
    assert torch.equal(y[:30], want[:30])  # (sequence 1 is empty, 2 is tokens 30 .. 63, in any order with 0's)


@pytest.mark.parametrize("qb", [16, 32, 64, 128])
@pytest.mark.parametrize("hd,nh,nkv", [(64, 2, 2), (32, 4, 1), (128, 2, 1), (80, 1, 1)])
def test_blocks(hip, qb, hd, nh, nkv):
    import torch
    rng = np.random.default_rng(qb + hd)
    lens, keys = [700, 1, 64, 0, 333, 129], [700, 1, 0, 0, 300, 65]
    x = _codes(rng, sum(lens), (nh + 2 * nkv) * hd)
    start = _starts(lens)
    for top_k, key_len, xl in ((1, None, 0), (3, keys, T), (20, None, 0)):
        st = torch.from_numpy(start).cuda()
        kl = None if key_len is None else torch.tensor(key_len, dtype=torch.int32, device="cuda")
        got = hip.select_blocks(_dev(hip, x, xl), st, 700, nh, hd, top_k, n_kv_heads=nkv, query_block=qb, key_len=kl,
                                x_layout=xl, m_tokens=len(x))
        torch.cuda.synchronize()
        lists = ref.select(x, start, nh, nkv, hd, top_k, 700, qb, key_len)
        assert np.array_equal(got.cpu().numpy(), lists), (top_k, xl)
        for kind in (1, 3):
            _check(hip, x, lens, nh, nkv, hd, kind, xl, key_len=key_len, lists=lists, qb=qb, say=f"top {top_k}")


def test_all_blocks_listed_is_dense(hip):
    import torch
    x = torch.from_numpy(_codes(np.random.default_rng(4), 500, 3 * 2 * 64)).cuda()
    start = torch.tensor([0, 300, 500], dtype=torch.int32, device="cuda")
    blocks = hip.select_blocks(x, start, 300, 2, 64, 9)
    a = hip.attention(x, 0.04, start, 300, 2, 64, kind=1, blocks=blocks)
    b = hip.attention(x, 0.04, start, 300, 2, 64, kind=1)
    assert float((a - b).abs().max()) <= 2.0 ** -18 * 128 * 0.04


def test_lists_with_gaps_and_strangers(hip):
    """-1, numbers past the sequence's blocks and lists of nothing."""
    rng = np.random.default_rng(6)
    x = _codes(rng, 400, 3 * 64)
    lists = np.full((2, 1, 4, 3), -1, np.int32)
    lists[0, 0, 0], lists[0, 0, 1], lists[0, 0, 2] = [-1, 3, 1000], [0, -7, 2], [-1, -1, -1]
    lists[1, 0, 0], lists[1, 0, 1] = [2, 0, 1], [99, 98, 1]
    lists[0, 0, 3] = [1, 2 ** 31 - 1, -2 ** 31]
    for kind in (1, 3):
        got = _check(hip, x, [220, 180], 1, 1, 64, kind, lists=lists, max_len=220)
        assert not got[128:192].any()


def test_ties_go_to_the_lowest_block(hip):
    import torch
    x = np.zeros((64 * 9, 3 * 64), np.int8)
    x[:, :64], x[:, 64:128] = 1, 5
    x[64 * 4:64 * 5, 64:128] = 7
    st = torch.tensor([0, len(x)], dtype=torch.int32, device="cuda")
    got = hip.select_blocks(torch.from_numpy(x).cuda(), st, len(x), 1, 64, 3).cpu().numpy()
    assert (got == np.array([0, 1, 4])).all()


def test_scores_at_the_end_of_their_range(hip):
    import torch
    for qv, kv in ((-128, -128), (127, -128), (-128, 127)):
        x = np.zeros((64 * 6 + 1, 3 * 128), np.int8)
        x[:, :128], x[:, 128:256] = qv, kv
        x[64 * 3:64 * 4, 128] = 0
        st = np.array([0, len(x)], np.int32)
        got = hip.select_blocks(torch.from_numpy(x).cuda(), torch.from_numpy(st).cuda(), len(x), 1, 128, 4,
                                query_block=128).cpu().numpy()
        assert np.array_equal(got, ref.select(x, st, 1, 1, 128, 4, len(x), 128))


@pytest.mark.parametrize("n", [64 * 300, 64 * 1100 + 5])
def test_many_blocks(hip, n):
    """More blocks than a lane's first few hold."""
    import torch
    rng = np.random.default_rng(n)
    x = _codes(rng, n, 3 * 32)
    st = np.array([0, n], np.int32)
    got = hip.select_blocks(torch.from_numpy(x).cuda(), torch.from_numpy(st).cuda(), n, 1, 32, 40, query_block=128)
    assert np.array_equal(got.cpu().numpy(), ref.select(x, st, 1, 1, 32, 40, n, 128))


def test_offsets_past_32_bits(hip):
    """A sequence that lies beyond 4 GiB of codes."""
    import torch
    cols, m = 3 * 12 * 64, 2000000
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GiB of free GPU memory")
    part = _codes(np.random.default_rng(3), 333, cols)
    x = torch.zeros((m, cols), dtype=torch.int8, device="cuda")
    x[m - 333:] = torch.from_numpy(part).cuda()
    start = torch.tensor([m - 333, m], dtype=torch.int32, device="cuda")
    y = torch.zeros((m, 768), dtype=torch.float32, device="cuda")
    hip.attention(x, 0.04, start, 333, 12, 64, kind=1, out=y)
    blocks = hip.select_blocks(x, start, 333, 12, 64, 2)
    want = hip.attention(torch.from_numpy(part).cuda(), 0.04, torch.tensor([0, 333], dtype=torch.int32, device="cuda"),
                         333, 12, 64, kind=1)
    assert torch.equal(y[m - 333:], want) and not y[:m - 333].any()
    assert np.array_equal(blocks.cpu().numpy(), ref.select(part, np.array([0, 333]), 12, 12, 64, 2, 333, 64))
    del x, y
    torch.cuda.empty_cache()


def test_graph_and_stream(hip):
    import torch
    rng = np.random.default_rng(7)
    x = torch.from_numpy(_codes(rng, 800, 3 * 2 * 64)).cuda()
    start = torch.tensor([0, 500, 800], dtype=torch.int32, device="cuda")

    def step():
        b = hip.select_blocks(x, start, 500, 2, 64, 3)
        return b, hip.attention(x, 0.04, start, 500, 2, 64, kind=1, blocks=b), hip.attention(
            x, 0.04, start, 500, 2, 64, out_scale=0.02)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        x.copy_(torch.from_numpy(_codes(rng, 800, 3 * 2 * 64)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))
    st = torch.cuda.Stream()  # a stream given by hand
    st.wait_stream(torch.cuda.current_stream())
    b = hip.select_blocks(x, start, 500, 2, 64, 3, stream=st)
    y = hip.attention(x, 0.04, start, 500, 2, 64, kind=1, blocks=b, stream=st)
    st.synchronize()
    assert torch.equal(y, out[1])


def test_a_block_listed_twice_counts_twice(hip):
    """Weights of a block's keys double, of the short last one too."""
    import torch
    x = _codes(np.random.default_rng(12), 150, 3 * 64)
    xs, start = float(np.float32(0.03)), np.array([0, 150])
    lists = np.array([[[[0, 2, 0, 2, 2], [1, 1, 0, -1, -1], [2, 2, -1, 2, 0]]]], np.int32)
    got = hip.attention(torch.from_numpy(x).cuda(), xs, torch.tensor([0, 150], dtype=torch.int32, device="cuda"), 150, 1,
                        64, kind=1, blocks=torch.from_numpy(lists).cuda()).cpu().numpy()
    q, k, v = (t[:, 0] for t in ref.split_heads(x, start, 0, 1, 1, 64))
    times = np.array([[np.sum(lists[0, 0, i // 64] == j // 64) for j in range(150)] for i in range(150)])
    z = q @ k.T * (xs * xs / 8)
    p = times * np.exp(z - z.max(1, keepdims=True))
    want = (p / p.sum(1, keepdims=True)) @ v * xs
    spread = 1.45 * float((z.max(1) - z.min(1)).max())
    rel = 2.0 ** -23 + spread * (2.0 ** -23 + 2.0 ** -22) + 2.0 ** -20  # as in the bars above
    assert np.abs(got - want).max() <= 128 * xs * (2 * rel + (320 / 16 + 8) * 2.0 ** -24)


def test_select_on_two_streams(hip):
    """Each call's workspace is its stream's: two streams that choose at once do not meet in it."""
    import torch
    rng = np.random.default_rng(14)
    xs = [torch.from_numpy(_codes(rng, 4096, 3 * 2 * 64)).cuda() for _ in range(2)]
    start = torch.tensor([0, 4096], dtype=torch.int32, device="cuda")
    want = [hip.select_blocks(x, start, 4096, 2, 64, 8) for x in xs]
    outs = [[torch.empty_like(want[0]) for _ in range(20)] for _ in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for i in range(20):
        for x, st, o in zip(xs, streams, outs):
            hip.select_blocks(x, start, 4096, 2, 64, 8, out=o[i], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for o, w in zip(outs, want) for t in o)


@pytest.mark.parametrize("kind", [1, 3])
def test_growing_scores_in_every_shape(hip, kind):
    """Keys whose scores grow to the end, so that m moves again and again, in the shapes that the sizes choose:
    two tiles a wave, keys split over waves, and the common one; one sequence shorter than a chunk among them."""
    rng = np.random.default_rng(21)
    for lens, nh in (([2048] * 4, 16), ([900], 2), ([300] * 40 + [7], 4)):
        x = _codes(rng, sum(lens), 3 * nh * 64)
        grow = np.concatenate([np.linspace(0.02, 1.0, n) for n in lens])[:, None]
        keys = slice(nh * 64, 2 * nh * 64)
        x[:, keys] = np.clip(np.rint(x[:, keys] * grow * 2), -127, 127).astype(np.int8)
        _check(hip, x, lens, nh, nh, 64, kind, x_scale=0.15)


@pytest.mark.parametrize("qb", [16, 32, 64, 128])
@pytest.mark.parametrize("hd", [32, 64, 96, 128])
def test_lists_in_every_shape(hip, qb, hd):
    """Few workgroups (a list's keys split over waves) and many, with lists of numbers out of order, gaps and a short
    last block, and with scores that grow."""
    rng = np.random.default_rng(qb + hd)
    for lens, nh in (([450, 0, 70], 2), ([200, 65, 1, 130] * 40, 4)):
        x = _codes(rng, sum(lens), 3 * nh * hd)
        keys = slice(nh * hd, 2 * nh * hd)
        grow = np.concatenate([np.linspace(0.1, 1.0, n) for n in lens])[:, None]
        x[:, keys] = np.clip(np.rint(x[:, keys] * grow * 2), -127, 127).astype(np.int8)
        for top_k in (3, 6):
            order = rng.permuted(np.tile(np.arange(8), (len(lens), nh, -(-max(lens) // qb), 1)), axis=-1)
            lists = np.where(order < 7, order, -1)[..., :top_k]
            _check(hip, x, lens, nh, nh, hd, 1 if top_k == 3 else 3, x_scale=0.1, lists=lists, qb=qb)


@pytest.mark.parametrize("hd", [32, 96, 128])
def test_growing_scores_in_every_shape_of_other_heads(hip, hd):
    """Few long sequences (keys split over waves), many, and one with too few keys for all of the parts."""
    rng = np.random.default_rng(hd)
    for lens, nh, kind in (([900], 2, 1), ([2100], 3, 3), ([300] * 40 + [7], 4, 1), ([300, 20], 1, 3)):
        x = _codes(rng, sum(lens), 3 * nh * hd)
        grow = np.concatenate([np.linspace(0.02, 1.0, n) for n in lens])[:, None]
        keys = slice(nh * hd, 2 * nh * hd)
        x[:, keys] = np.clip(np.rint(x[:, keys] * grow * 2), -127, 127).astype(np.int8)
        _check(hip, x, lens, nh, nh, hd, kind, x_scale=0.1)
