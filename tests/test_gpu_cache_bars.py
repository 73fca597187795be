"""cache_attention against its definition in 64 bits with the bars of cache_bars.py, the same for fp32 results and int8
codes, of which at most 5e-4 may differ from the definition's: both kernels, every head size, keys in one part and in
several, sequences in order of length, weights flat and far apart."""
import numpy as np
import pytest

import attention_bars
import cache_bars as bars
from test_gpu_cache import FILL, Batch, codes

pytestmark = pytest.mark.gpu


def check(hip, rng, b, nh, form, kind, causal=True, qs=0.04, ks=0.05, vs=0.03, parts=1):
    import torch
    hd, f, q = b.hd, lambda v: float(np.float32(v)), codes(rng, b.m, nh * b.hd)  # noqa: E731
    print(f"cache_attention {b.news[:6]} over {b.lens[:6]} heads={nh}/{b.nkv}x{hd} kind={kind} causal={causal}", flush=True)
    scale = f(qs) * f(ks) * f(hd ** -0.5)
    want, bar, real = bars.attention(q, b.cache, b.start, b.len, b.table, nh, scale, causal, form, parts)
    want, bar = want[real] * f(vs), bar[real] * f(vs)
    so = attention_bars.output_scale(want)
    out = torch.full((b.m, nh * hd), FILL, dtype=torch.float32 if kind == 1 else torch.int8, device="cuda")
    hip.cache_attention(torch.from_numpy(q).cuda(), *b.dev, b.most_new, b.longest, nh, q_scale=qs, k_scale=ks, v_scale=vs,
                        causal=causal, kind=kind, out_scale=so, out=out)
    torch.cuda.synchronize()
    assert hip.last_path() == f"cache {form} {hd},{parts}"
    got = out.cpu().numpy()
    assert (got[~real] == FILL).all()
    attention_bars.assert_within(got[real], want, bar, so if kind == 3 else None)


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("hd", range(16, 129, 16))
@pytest.mark.parametrize("causal", [True, False])
def test_every_head_size(hip, hd, kind, causal):
    rng = np.random.default_rng([hd, kind])
    check(hip, rng, Batch(hip, rng, [1, 2, 1, 5], [256, 100, 17, 66], 16, 2, hd, gap=2), 8, "split", kind, causal)
    check(hip, rng, Batch(hip, rng, [40, 64, 1, 130, 3] * 6, [40, 200, 70, 130, 2] * 6, 16, 6, hd, gap=2), 12, "prompt", kind,
          causal)


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("news,lens,nh,nkv,hd,parts", [
    ([1], [2000], 8, 8, 64, 4), ([1, 1], [1300, 900], 32, 8, 128, 3), ([4, 1, 2], [5000, 40, 2600], 4, 2, 64, 10),
    ([2], [40000], 8, 1, 64, 79)])
def test_few_queries_in_parts(hip, kind, news, lens, nh, nkv, hd, parts):
    rng = np.random.default_rng([sum(lens), nh, kind])
    check(hip, rng, Batch(hip, rng, news, lens, 64, nkv, hd), nh, "split", kind, parts=parts)


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("news,lens,nh,nkv,hd,parts", [
    ([300, 1], [2300, 900], 40, 20, 64, 2), ([129, 40, 7], [1500, 1300, 7], 64, 16, 128, 2), ([500], [500], 40, 40, 32, 1)])
@pytest.mark.parametrize("causal", [True, False])
def test_many_queries(hip, kind, news, lens, nh, nkv, hd, parts, causal):
    rng = np.random.default_rng([sum(lens), nh, kind])
    check(hip, rng, Batch(hip, rng, news, lens, 64, nkv, hd), nh, "prompt", kind, causal, parts=parts)


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("form,new", [("split", 1), ("prompt", 40)])
@pytest.mark.parametrize("qs,ks", [(1e-20, 1e-20), (1e-3, 1e-2), (0.5, 0.5), (3.0, 2.0), (1e3, 1e3)])
def test_scales(hip, kind, form, new, qs, ks):
    """Flat weights, and rows where one key has all of it."""
    rng = np.random.default_rng([new, kind])
    b = Batch(hip, rng, [new] * 5, [400, 300, 90, 64, new], 16, 26, 64)
    check(hip, rng, b, 26, form, kind, qs=qs, ks=ks)
