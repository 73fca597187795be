"""Scales at the ends of what 32-bit floats hold. A code is clamp(rint(value / scale)) whatever the size of the quotient: 0
where the value is 0, though the quotient's factor is more than a float; and a mean of values keeps its accuracy where
their scale over the sum of the weights is less than one. Bars: test_gpu_cache.py's; a result of a scale below 2^-126
* 2^24 also ends at a step of 2^-149."""
import numpy as np
import pytest

import cache_ref as ref
from test_gpu_cache import TOL, Batch, codes

pytestmark = pytest.mark.gpu


def cuda(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("x_type,xs,scale", [("i8", 1e25, 1e-20), ("i8", 3e38, 1e-45), ("f32", 1.0, 1e-39), ("f32", 1.0, 1e-45)])
def test_append_far_apart(hip, new, x_type, xs, scale):
    rng = np.random.default_rng(new)
    b = Batch(hip, rng, [new, new], [new + 3, new], 16, 2, 32)
    x = rng.integers(-1, 2, (b.m, 6 * 32)).astype(np.int8)
    q = hip.cache_append(cuda(x if x_type == "i8" else x.astype(np.float32)), *b.dev, new, 2, x_scale=xs, q_scale=scale,
                         k_scale=scale, v_scale=scale)
    want = 127 * x.astype(np.int64)
    assert np.array_equal(q.cpu().numpy(), want[:, :64])
    cache = b.dev[0].cpu().numpy()
    _, stored = ref.append(want.astype(np.float64), b.start, b.len, b.table, 16, b.n_pages, 2, 2, 32, ref.NONE, None, 1.0)
    assert len(stored) == b.m
    for page, place, k, v in stored:
        for h in range(2):
            assert np.array_equal(ref.key_of(cache, page, h, place), k[h])
            assert np.array_equal(ref.value_of(cache, page, h, place), v[h])


def attend(hip, b, q, kind, vs, so, longest):
    y = hip.cache_attention(cuda(q), *b.dev, b.most_new, longest, 2, q_scale=0.04, k_scale=0.05, v_scale=vs,
                            kind=hip.EPI_F32 if kind == "f32" else hip.EPI_I8, out_scale=so).cpu().numpy()
    want, _ = ref.attention(q, b.cache, b.start, b.len, b.table, 2,
                            float(np.float32(0.04)) * float(np.float32(0.05)) * float(np.float32(64 ** -0.5)), True)
    return y, np.stack([want[t].reshape(-1) for t in range(b.m)])


# few queries and many, and either with keys in parts
FORMS = [([1, 1], [0, 70], 100), ([1, 1, 1], [0, 70, 3000], 3000), ([200, 1], [60, 300], 300), ([40, 3], [20, 4000], 4000)]


@pytest.mark.parametrize("news,lens,longest", FORMS)
@pytest.mark.parametrize("vs,so", [(0.03, 1e-39), (0.03, 1e-45), (1e10, 1e-38), (3e38, 1e-45), (3e38, 3e-38), (1e-30, 1e-45)])
def test_codes_of_large_quotients(hip, news, lens, longest, vs, so):
    rng = np.random.default_rng(len(news))
    b = Batch(hip, rng, news, lens, 16, 2, 64)
    b.cache[:, 1, 0] = 0  # (values of the first head: all 0)
    b.dev[0] = cuda(b.cache)
    y, want = attend(hip, b, codes(rng, b.m, 128), "i8", vs, so, longest)
    assert (want[:, :64] == 0).all() and (y[:, :64] == 0).all()
    assert np.array_equal(y[:, 64:], 127 * np.sign(want[:, 64:]))
    assert (want[:, 64:] == 0).any()  # (queries that see nothing)


@pytest.mark.parametrize("news,lens,longest", FORMS)
@pytest.mark.parametrize("kind", ["f32", "i8"])
@pytest.mark.parametrize("vs", [1e-30, 1e-34, 1e-37, 1e-40, 1e36])
def test_small_and_large_values(hip, news, lens, longest, kind, vs):
    rng = np.random.default_rng(len(news) + 10)
    b = Batch(hip, rng, news, lens, 16, 2, 64)
    f = lambda v: float(np.float32(v))  # noqa: E731
    y, want = attend(hip, b, codes(rng, b.m, 128) // 16, kind, vs, vs, longest)
    if kind == "f32":
        assert np.abs(y.astype(np.float64) - want * f(vs)).max() <= TOL * f(vs) + 2.0 ** -149
    else:
        assert np.abs(y - want).max() <= 0.5 + TOL + 1e-3
