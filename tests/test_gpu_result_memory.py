"""Results that a call allocates where it runs on a stream that is not the current one: their memory has no work of the
current stream under way on it, and is not handed on while the current stream's work on the result is."""
import numpy as np
import pytest

from test_gpu_cache import Batch, codes

pytestmark = pytest.mark.gpu

M = 20000  # (results of a size of their own in torch's allocator: over 1 MB)


def cuda(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def append(hip, rng):
    b = Batch(hip, rng, [M], [M], 16, 1, 64)
    x = cuda(codes(rng, b.m, 4 * 64))
    return lambda s: (hip.cache_append(x, *b.dev, M, 2, x_scale=0.03, q_scale=0.03, k_scale=0.04, v_scale=0.03, stream=s),)


def attend(kind, y_layout=0):
    def make(hip, rng):
        b = Batch(hip, rng, [1] * M, [1] * M, 16, 1, 64)
        q = cuda(codes(rng, b.m, 2 * 64))
        return lambda s: (hip.cache_attention(q, *b.dev, 1, 1, 2, q_scale=0.04, k_scale=0.05, v_scale=0.03, kind=kind,
                                              out_scale=0.04, y_layout=y_layout, stream=s),)
    return make


def linear(kind, y_layout=0):
    def make(hip, rng):
        w = rng.integers(-8, 9, (64, 64)).astype(np.int8)
        packed = hip.PackedWeight.pack(w, np.full(64, 0.01, np.float32))
        x = cuda(codes(rng, M, 64))
        return lambda s: (packed.run(x, 0.05, kind, out_scale=0.05, y_layout=y_layout, stream=s),)
    return make


def quantize(layout):
    def make(hip, rng):
        x = cuda(rng.standard_normal((M, 64)).astype(np.float32))
        return lambda s: (hip.quantize_act(x, 0.03, layout=layout, stream=s),)
    return make


def norm(hip, rng):
    y, r = (cuda(rng.standard_normal((M, 64)).astype(np.float32)) for _ in range(2))
    gamma, beta = (cuda(rng.standard_normal(64).astype(np.float32)) for _ in range(2))
    return lambda s: hip.residual_norm(y, gamma, beta, residual=r, keep_sum=True, keep_norm=True, out_scale=0.03, stream=s)


def encoder(kind):
    def make(hip, rng):
        x, start = cuda(codes(rng, M, 3 * 128)), cuda(np.arange(0, M + 1, 50, dtype=np.int32))
        return lambda s: (hip.attention(x, 0.03, start, 50, 2, 64, kind=kind, out_scale=0.03, stream=s),)
    return make


def select(hip, rng):
    x, start = cuda(codes(rng, M, 3 * 128)), cuda(np.arange(0, M + 1, 400, dtype=np.int32))
    return lambda s: (hip.select_blocks(x, start, 400, 2, 64, 200, query_block=16, stream=s),)


CALLS = {"run, fp32": linear(1), "run, codes": linear(3), "run, blocks": linear(3, 1), "quantize_act": quantize(0),
         "quantize_act, blocks": quantize(1), "residual_norm": norm, "attention, fp32": encoder(1),
         "attention, codes": encoder(3), "select_blocks": select, "cache_append": append, "cache_attention, codes": attend(3), "cache_attention, blocks": attend(3, 1),
         "cache_attention, fp32": attend(1)}


@pytest.mark.parametrize("name", CALLS)
def test_results_on_another_stream(hip, name):
    import torch
    call = CALLS[name](hip, np.random.default_rng(1))
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    sizes = [(t.shape, t.dtype) for t in want]
    torch.cuda.empty_cache()
    # memory of the results' sizes that is free again, with work of the current stream still to come on it
    free = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in sizes]
    before = {t.data_ptr() for t in free}
    torch.cuda._sleep(20_000_000)
    for t in free:
        t.fill_(1)
    del t, free
    got = call(s)
    assert not before & {t.data_ptr() for t in got}
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    # the current stream reads the results late; the next ones are elsewhere until then
    at = {t.data_ptr() for t in got}
    torch.cuda._sleep(20_000_000)
    late = [t.clone() for t in got]
    del got
    again = call(s)
    assert not at & {t.data_ptr() for t in again}
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(late, want)) and all(torch.equal(g, w) for g, w in zip(again, want))


@pytest.mark.parametrize("name", CALLS)
def test_results_on_the_current_stream_by_name(hip, name):
    """The current stream given as `stream` is no other stream: results are the current stream's own, handed on at once."""
    import torch
    call = CALLS[name](hip, np.random.default_rng(2))
    want = [t.clone() for t in call(None)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = call(s)
        at = {t.data_ptr() for t in got}
        kept = [t.clone() for t in got]
        del got
        assert {t.data_ptr() for t in call(s)} == at
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(kept, want))


@pytest.mark.parametrize("name", CALLS)
def test_results_on_another_stream_of_a_captured_graph(hip, name):
    """A call on a stream that a capture forks to, its results used where the streams meet; replayed several times, with
    eager work between."""
    import torch
    call = CALLS[name](hip, np.random.default_rng(3))
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        first = call(side)
        main.wait_stream(side)
        kept = [t.clone() for t in first]
        del first
        side.wait_stream(main)
        second = call(side)
        main.wait_stream(side)
    for _ in range(4):
        for t in (*kept, *second):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(k, w) and torch.equal(s, w) for k, s, w in zip(kept, second, want))
        assert all(torch.equal(t, w) for t, w in zip(call(None), want))
