"""cache_append and cache_attention as programs use them: other streams, two calls at once, graphs, repeated calls, shared
pages, caches and activations past 32-bit offsets, very many sequences, lengths out of range, and what the binding
refuses. Results are held to the bars of test_gpu_cache.py."""
import numpy as np
import pytest

import cache_ref as ref
from test_gpu_cache import DELTA, TOL, Batch, codes, run_append, run_attend

pytestmark = pytest.mark.gpu


def cuda(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def attend(hip, q, b, nh, **more):
    return hip.cache_attention(q, *b.dev, b.most_new, b.longest, nh, q_scale=0.04, k_scale=0.05, v_scale=0.03,
                               kind=hip.EPI_F32, **more)


def append(hip, x, b, nh, **more):
    return hip.cache_append(x, *b.dev, b.most_new, nh, x_scale=0.03, q_scale=0.03, k_scale=0.04, v_scale=0.03, **more)


@pytest.mark.parametrize("new", [1, 64])
def test_the_same_call_gives_the_same_bits(hip, new):
    import torch
    rng = np.random.default_rng(1)
    b = Batch(hip, rng, [new, new], [5000, 1300], 64, 2, 64)
    q = cuda(codes(rng, b.m, 512))
    want = attend(hip, q, b, 8)
    for _ in range(5):
        assert torch.equal(attend(hip, q, b, 8), want)


@pytest.mark.parametrize("new", [1, 64])
def test_two_streams_at_once(hip, new):
    """Calls that need a workspace, on two streams that are not the current one."""
    import torch
    rng = np.random.default_rng(2)
    batches = [Batch(hip, rng, [new] * 2, [4000, 3500], 32, 2, 64) for _ in range(2)]
    qs = [cuda(codes(rng, b.m, 512)) for b in batches]
    want = [attend(hip, q, b, 8) for q, b in zip(qs, batches)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(attend(hip, qs[i], batches[i], 8, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_append_on_another_stream(hip):
    import torch
    rng = np.random.default_rng(3)
    b = Batch(hip, rng, [20, 1], [30, 9], 16, 2, 64)
    x = cuda(codes(rng, b.m, 8 * 64))
    clean = b.dev[0].clone()
    want_q, want = append(hip, x, b, 4), b.dev[0].clone()
    b.dev[0].copy_(clean)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    q = append(hip, x, b, 4, stream=s)
    s.synchronize()
    assert torch.equal(q, want_q) and torch.equal(b.dev[0], want)


@pytest.mark.parametrize("new", [1, 3, 40])
def test_captured_and_replayed(hip, new):
    """Lengths grow and pages are taken on the device between replays; eager work runs between them."""
    import torch
    rng = np.random.default_rng(4)
    lens0 = [2100, 17]
    b = Batch(hip, rng, [new] * 2, [n + 8 * new for n in lens0], 16, 2, 64)
    cache, table, start, lens = b.dev
    x = cuda(codes(rng, b.m, 8 * 64))
    freq = cuda((10000.0 ** (-np.arange(32) / 32)).astype(np.float32))
    first = cuda(np.array(lens0, np.int32))

    def step():
        q = append(hip, x, b, 4, rope=hip.ROPE_HALF, inv_freq=freq)
        return attend(hip, q, b, 4)

    def run(one):
        cache.copy_(cuda(b.cache))
        lens.copy_(first)
        out = []
        for _ in range(6):
            lens.add_(new)
            out.append(one().clone())
        return out, cache.clone()

    want, want_cache = run(step)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()

    def replay():
        graph.replay()
        torch.cuda.synchronize()
        attend(hip, cuda(codes(rng, b.m, 256)), b, 4)  # eager work between
        return y

    got, got_cache = run(replay)
    assert torch.equal(got_cache, want_cache)
    for w, g in zip(want, got):
        assert torch.equal(w, g)


def test_sequences_share_the_pages_of_a_prefix(hip):
    """Four sequences whose first 48 tokens lie in the same pages, each with pages of its own behind them."""
    rng = np.random.default_rng(5)
    b = Batch(hip, rng, [1, 1, 5, 1], [60, 70, 64, 49], 16, 2, 64)
    b.table[1:, :3] = b.table[0, :3]
    b.dev[1] = cuda(b.table)
    run_attend(hip, rng, b, 4)
    run_append(hip, rng, b, 4, "i8", ref.HALF)


@pytest.mark.parametrize("new", [1, 50])
def test_lengths_out_of_range(hip, new):
    """Starts outside the tokens are brought into range; lengths below 0 are none, and lengths past the pages of the table
    see what there is."""
    rng = np.random.default_rng(6)
    b = Batch(hip, rng, [new, new, new], [70, 70, 70], 16, 1, 32)
    b.dev[2] = cuda(np.array([-3, new, new, 2 ** 31 - 1], np.int32))
    b.start = np.array([0, new, new, b.m], np.int32)  # as the calls take them
    b.most_new = 2 * new
    run_attend(hip, rng, b, 2)
    run_append(hip, rng, b, 2, "i8", ref.HALF)
    b.len = np.array([-5, 3, 70 + 16 * 50], np.int32)
    b.dev[3] = cuda(b.len)
    b.cache = b.dev[0].cpu().numpy()
    for causal in (True, False):
        run_attend(hip, rng, b, 2, causal=causal)
    run_append(hip, rng, b, 2, "i8", ref.HALF)


def test_a_cache_past_32_bit_offsets(hip):
    """Pages beyond 4 GiB: 40000 of 128 KiB, of which the last ones are used."""
    import torch
    rng = np.random.default_rng(7)
    ps, nkv, hd, n_pages = 64, 8, 128, 40000
    small = Batch(hip, rng, [1, 40], [150, 100], ps, nkv, hd, spare=0)
    assert (n_pages - small.n_pages) * 2 * nkv * ps * hd > 2 ** 32
    cache = torch.zeros(hip.cache_shape(n_pages, ps, nkv, hd), dtype=torch.int8, device="cuda")
    base = n_pages - small.n_pages
    cache[base:] = small.dev[0]
    table = np.where(small.table >= 0, small.table + base, -1).astype(np.int32)
    dev = [cache, cuda(table), small.dev[2], small.dev[3]]
    x = cuda(codes(rng, small.m, (16 + 2 * nkv) * hd))
    q = append(hip, x, small, 16)
    want = attend(hip, q, small, 16)
    small.dev = dev
    q2 = append(hip, x, small, 16)
    got = attend(hip, q2, small, 16)
    assert torch.equal(q, q2) and torch.equal(got, want)
    assert not cache[:base].any()


def test_the_longest_sequence(hip):
    """As many tokens as a table may name, 2^31 - 65536: its first half all in one page, its second in another. (A wave adds
    up 2^31 / (512 parts * 4 waves * 64 keys) = 16384 spans, and a query's join under 200 parts: 2^-24 of the sum for each
    addition, in the numerator and in the denominator, is 2e-3 of the largest |v|.)"""
    import torch
    rng = np.random.default_rng(12)
    ps, hd, entries = 256, 16, 2 ** 23 - 256
    cache = codes(rng, *hip.cache_shape(2, ps, 1, hd))
    values = cache[:, 1, 0].reshape(2, ps // 16, hd, 16)  # (a view)
    values[0], values[1] = np.abs(values[0]), -np.abs(values[1])
    q = codes(rng, 1, hd)
    table = torch.zeros((1, entries), dtype=torch.int32, device="cuda")
    table[:, entries // 2:] = 1
    length = entries * ps
    y = hip.cache_attention(cuda(q), cuda(cache), table, cuda(np.array([0, 1], np.int32)), cuda(np.array([length], np.int32)),
                            1, length, 1, q_scale=0.04, k_scale=0.05, v_scale=0.03, kind=hip.EPI_F32)
    assert hip.last_path() == "cache split 16,512"
    z = cache[:, 0, 0].astype(np.float64) @ q[0] * (float(np.float32(0.04)) * float(np.float32(0.05)) / 4)
    w = np.exp(z - z.max())  # [2, ps], each key as often as any other
    v = values.astype(np.float64).transpose(0, 1, 3, 2).reshape(2, ps, hd)
    want = (w[..., None] * v).sum((0, 1)) / w.sum() * float(np.float32(0.03))
    bar = (2e-3 * 127 + TOL) * 0.03
    first = (w[0, :, None] * v[0]).sum(0) / w[0].sum() * 0.03
    assert np.abs(first - want).max() > 2 * bar
    assert np.abs(y.cpu().numpy() - want).max() <= bar


def test_activations_past_32_bit_offsets(hip):
    """The tokens of the last sequence lie beyond 4 GiB of fp32 x; only they belong to one."""
    import torch
    rng = np.random.default_rng(8)
    nh, nkv, hd = 8, 8, 128
    cols = (nh + 2 * nkv) * hd
    b = Batch(hip, rng, [30], [30], 16, nkv, hd)
    m = 2 ** 30 // cols + 400
    x = torch.zeros((m, cols), device="cuda")
    x[-30:] = torch.randn((30, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    assert (m - 30) * cols * 4 > 2 ** 32
    q = append(hip, x[-30:].clone(), b, nh)
    want = b.dev[0].clone()
    b.dev[0].zero_()
    b.dev[0].copy_(cuda(b.cache))
    b.dev[2] = cuda(np.array([m - 30, m], np.int32))
    q2 = append(hip, x, b, nh, out=torch.zeros((m, nh * hd), dtype=torch.int8, device="cuda"))
    assert torch.equal(q2[-30:], q) and torch.equal(b.dev[0], want) and not q2[:-30].any()
    y = attend(hip, q, Batch_like(b, [0, 30]), nh)
    y2 = attend(hip, q2, b, nh)
    assert torch.equal(y2[-30:], y)


def Batch_like(b, start):
    """The same batch with other starts."""
    import copy
    c = copy.copy(b)
    c.dev = list(b.dev)
    c.dev[2] = cuda(np.array(start, np.int32))
    return c


def test_more_sequences_than_a_launch_has_rows(hip):
    """70000 sequences of one token over 1 or 2: several launches."""
    import torch
    rng = np.random.default_rng(9)
    n, ps, hd = 70000, 16, 16
    cache = cuda(codes(rng, *hip.cache_shape(n, ps, 1, hd)))
    table = cuda(rng.permutation(n).astype(np.int32)[:, None])
    start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    lens = cuda(rng.integers(1, 3, n).astype(np.int32))
    x = cuda(codes(rng, n, 3 * hd))
    q = hip.cache_append(x, cache, table, start, lens, 1, 1, x_scale=0.03, q_scale=0.03, k_scale=0.03, v_scale=0.03)
    assert torch.equal(q, x[:, :hd])
    y = hip.cache_attention(q, cache, table, start, lens, 1, 2, 1, q_scale=0.04, k_scale=0.05, v_scale=0.03, kind=hip.EPI_F32)
    pages = cache[table[:, 0].long()]
    at, slot = torch.arange(n, device="cuda"), lens.long() - 1
    assert torch.equal(pages[at, 0, 0, slot], x[:, hd:2 * hd])
    values = pages[:, 1, 0].reshape(n, 1, hd, 16)[:, 0].transpose(1, 2)[:, :2].double()  # [n, 2, hd]
    assert torch.equal(values[at, slot], x[:, 2 * hd:].double())
    z = (pages[:, 0, 0, :2].double() * q[:, None].double()).sum(2) * (float(np.float32(0.04)) * float(np.float32(0.05)) / 4)
    z[lens == 1, 1] = -np.inf
    want = (torch.softmax(z, 1)[..., None] * values).sum(1) * float(np.float32(0.03))
    assert float((y - want).abs().max()) <= TOL * 0.03


def test_what_the_binding_refuses(hip):
    import torch
    rng = np.random.default_rng(10)
    b = Batch(hip, rng, [2, 1], [5, 3], 16, 2, 64)
    x, q = cuda(codes(rng, b.m, 8 * 64)), cuda(codes(rng, b.m, 256))
    good = list(b.dev)

    def refused(call, **change):
        b.dev = [change.get(n, t) for n, t in zip(("cache", "table", "start", "lens"), good)]
        with pytest.raises(ValueError):
            call()
        b.dev = good

    for call in (lambda: append(hip, x, b, 4), lambda: attend(hip, q, b, 4)):
        refused(call, cache=good[0].cpu())
        refused(call, cache=good[0].float())
        refused(call, cache=good[0][:, :1])
        refused(call, cache=good[0].transpose(2, 3))
        refused(call, table=good[1].long())
        refused(call, table=good[1][:1])
        refused(call, table=good[1].t())
        refused(call, start=good[2][:-1])
        refused(call, start=good[2].cpu())
        refused(call, lens=good[3].long())
        refused(call, lens=good[3][:1])
    refused(lambda: append(hip, x.cpu(), b, 4))
    refused(lambda: append(hip, x[:, :-1], b, 4))
    refused(lambda: append(hip, x.double(), b, 4))
    refused(lambda: append(hip, x, b, 5))
    refused(lambda: append(hip, x, b, 4, rope=hip.ROPE_HALF))
    refused(lambda: append(hip, x, b, 4, rope=hip.ROPE_HALF, inv_freq=torch.ones(32, dtype=torch.float64, device="cuda")))
    refused(lambda: append(hip, x, b, 4, rope=hip.ROPE_HALF, inv_freq=torch.ones(32, device="cuda"),
                           positions=torch.zeros(2, dtype=torch.int32, device="cuda")))
    refused(lambda: append(hip, x, b, 4, x_layout=hip.LAYOUT_T16X32, m_tokens=b.m))
    refused(lambda: append(hip, x, b, 4, out=torch.empty((b.m, 255), dtype=torch.int8, device="cuda")))
    refused(lambda: attend(hip, q.cpu(), b, 4))
    refused(lambda: attend(hip, q.float(), b, 4))
    refused(lambda: attend(hip, q[:, :128].contiguous(), b, 4))
    refused(lambda: attend(hip, q, b, 4, m_tokens=b.m + 1))
    refused(lambda: attend(hip, q, b, 4, out=torch.empty((b.m, 256), dtype=torch.int8, device="cuda")))
    with pytest.raises(hip.SparseLinearError):
        append(hip, x, b, 4, rope=hip.ROPE_HALF, inv_freq=torch.ones(33, device="cuda"))  # more than half a head
    with pytest.raises(hip.SparseLinearError):
        attend(hip, q, b, 4, softmax_scale=-1.0)
    with pytest.raises(hip.SparseLinearError):  # heads of no features
        b.dev = [good[0][..., :0].contiguous(), *good[1:]]
        attend(hip, q, b, 4)
    b.dev = good


def test_nothing_to_do(hip):
    import torch
    rng = np.random.default_rng(11)
    b = Batch(hip, rng, [2], [5], 16, 2, 64)
    before = b.dev[0].clone()
    b.dev[2] = cuda(np.zeros(2, np.int32))
    q = append(hip, torch.empty((0, 8 * 64), dtype=torch.int8, device="cuda"), b, 4)
    y = attend(hip, q, b, 4)
    assert q.shape == (0, 256) and y.shape == (0, 256) and torch.equal(b.dev[0], before)


def test_bars():
    assert DELTA == 1e-3 and TOL == 4e-5 * 127
