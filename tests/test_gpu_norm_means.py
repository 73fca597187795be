"""GPU tests of residual_norm where the spread of a row is small against its mean:
LayerNorm's mean must be good to the row's spread, not to its values' own bits.

Bars, with u32 = 2^-24 and D = 100 as in test_gpu_residual_norm.py. A mean is off by
D u32 |mean| at most; taking the mean of the deviations from it off again, as is done
where the mean is over 4 deviations (every row here), leaves (D u32)^2 |mean|. For
values within a factor of 2 of their mean a difference is exact, so an element is off
by that times rstd |gamma|, and by (D + 10) u32 (|u| + |beta|) as any other. The
variance is off by at most 2 D u32 (var + (D u32 mean)^2), rstd by half of that over
var + eps. The row's fp32 values are the inputs: the definition in 64 bits has the
same ones."""
import numpy as np
import pytest

import encoder_ref as ref

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
D = 100


def check(hip, x, eps, post=False):
    """LayerNorm of fp32 rows x, as the only norm or as the one of the block's output."""
    import torch
    rng = np.random.default_rng(x.shape)
    g, b = (rng.normal(m, 0.3, x.shape[1]).astype(np.float32) for m in (1, 0))
    xd, gd, bd = (torch.from_numpy(a).cuda() for a in (x, g, b))
    if post:
        got = hip.residual_norm(xd, norm=hip.NORM_NONE, eps=eps, post_norm=hip.NORM_LAYER, post_gamma=gd, post_beta=bd,
                                keep_sum=True)[0].cpu().numpy()
    else:
        got = hip.residual_norm(xd, gd, bd, eps=eps, keep_norm=True)[1].cpu().numpy()
    x, g, b = (a.astype(np.float64) for a in (x, g, b))
    want = ref.norm_rows(x, 1, g, b, eps)
    mean, var = x.mean(1, keepdims=True), x.var(1, keepdims=True)
    far = np.abs(x - mean).max(1, keepdims=True) / np.sqrt(var + eps)
    rel = D * U32 * (var + (D * U32 * mean) ** 2) / (var + eps)
    bar = ((D * U32) ** 2 * np.abs(mean) / np.sqrt(var + eps) + far * rel) * np.abs(g).max()
    bar = bar + (D + 10) * U32 * (far * np.abs(g).max() + np.abs(b).max())
    over = np.abs(got - want) - bar
    assert np.isfinite(got).all() and over.max() <= 0, f"{x.shape}: {np.abs(got - want).max()} off, bar {bar.max()}"


WIDTHS = [1, 2, 3, 7, 31, 100, 257, 300, 511, 768, 1000, 1001, 1024, 1500, 2051, 3013, 4001, 5001, 16388, 65535]


@pytest.mark.parametrize("n", WIDTHS)
def test_rows_of_one_value(hip, n):
    """The definition gives beta, with the smallest eps in use; sums that fp32 holds exactly, and others."""
    values = np.array([100, 3, -12.5, 1, 0.1, 100.3, -7.77, 1 / 3, 1e-3], np.float32)
    x = np.repeat(values[:, None], n, 1)
    for post in (False, True):
        check(hip, x, 1e-12, post)


def test_many_rows_of_one_value(hip):
    """One wave a row."""
    for n in (1000, 777, 520):
        check(hip, np.repeat(np.linspace(-50, 50, 3000, dtype=np.float32)[:, None], n, 1), 1e-12)


@pytest.mark.parametrize("n", WIDTHS[3:])
def test_means_far_over_the_spread(hip, n):
    rng = np.random.default_rng(n)
    for mean in (10.0, 1000.0, -30000.0):
        x = (mean + rng.normal(0, 1, (9, n))).astype(np.float32)
        for post in (False, True):
            check(hip, x, 1e-6, post)


def test_not_a_number_in_a_row(hip):
    """As before, a row with one has nothing else, and the others do not see it."""
    import torch
    for n in (300, 768, 1001, 5000):
        x = torch.randn((6, n), device="cuda") + 50
        clean = hip.residual_norm(x, keep_norm=True)[1]
        x[1, n // 2], x[3, 0], x[4, n - 1] = float("nan"), float("inf"), float("-inf")
        got = hip.residual_norm(x, keep_norm=True)[1]
        assert torch.isnan(got[[1, 3, 4]]).all() and torch.equal(got[[0, 2, 5]], clean[[0, 2, 5]])
