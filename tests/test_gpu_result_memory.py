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


CALLS = {"cache_append": append, "cache_attention, codes": attend(3), "cache_attention, blocks": attend(3, 1),
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
        at = [t.data_ptr() for t in got]
        kept = [t.clone() for t in got]
        del got
        assert [t.data_ptr() for t in call(s)] == at
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(kept, want))
