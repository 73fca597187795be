"""The encoder of examples/encoder.py: every operator of a layer on what the one
before it left on the GPU, against the oracle (linears, quantisation) and the
64-bit definitions (attention, norms); and the whole against the same network in
fp32.

Bars. Linears as in test_gpu_parity.py. Attention and norms: an int8 code within
half a step, and fp32 values within 1e-5 of the largest, of the 64-bit value of
the same inputs (their own tests derive finer ones). Whole network: one int8
rounding moves an activation by step / sqrt(12) = max / 127 / 3.46, under 1.4 %
of its root mean square where the largest is up to 6 times that; a layer has five,
so two layers stay under 15 % even if all of them add up. Chosen blocks follow the
rounded codes, so with lists only the operators are compared.
"""
import os
import sys

import numpy as np
import pytest

import encoder_ref as ref
import oracle
from test_gpu_parity import check

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("lens,top_k", [([128, 1, 77, 300, 16], 0), ([700, 130], 3)])
def test_layers(hip, lens, top_k):
    import torch
    from encoder import Encoder, batch_of
    hidden, inter, heads = 256, 512, 4
    m, d = sum(lens), hidden // heads
    enc = Encoder(layers=2, hidden=hidden, inter=inter, heads=heads, sparsity=0.7)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((m, hidden), device="cuda", generator=g)
    want = enc.calibrate(x, lens, top_k)
    start, longest = batch_of(lens)
    seen = []
    got = enc(x, start, longest, top_k, tap=lambda i, r: seen.append(r))
    torch.cuda.synchronize()
    rows = lambda t, cols: hip.from_t16x32(t.cpu().numpy(), m, cols)  # noqa: E731
    st = start.cpu().numpy()
    for i, r in enumerate(seen):
        layer, c, nxt = enc.layers[i], enc.scales[i], enc.scales[i + 1]["x"]
        f = lambda v: np.float32(v)  # noqa: E731

        def linear(name, xin, cols, sx, kind, out, so=None):
            w = layer.dense[name]
            ref_y = oracle.linear(rows(xin, cols), w["w"], f(sx), w["sw"], w["b"], kind, **({} if so is None else {"so": f(so)}))
            y = rows(out, w["w"].shape[0]) if out.dtype == torch.int8 else out.cpu().numpy()
            check(kind, y, ref_y, f"layer {i} {name}")

        linear("qkv", r["xq"], hidden, c["x"], hip.EPI_I8, r["qkv"], c["qkv"])
        qkv = rows(r["qkv"], 3 * hidden)
        lists = None
        if top_k:
            lists = ref.select(qkv, st, heads, heads, d, top_k, longest, 64)
            assert np.array_equal(r["lists"].cpu().numpy(), lists)
        a, _ = ref.attention(qkv, float(f(c["qkv"])), st, heads, heads, d, d ** -0.5, lists=lists)
        off = np.abs(rows(r["att"], hidden) - np.clip(a / float(f(c["att"])), -127, 127))
        assert off.max() <= 0.5 + 1e-2, off.max()
        linear("out", r["att"], hidden, c["att"], hip.EPI_F32, r["y"])
        linear("ffn1", r["midq"], hidden, c["mid"], hip.EPI_I8_GELU, r["act"], c["act"])
        linear("ffn2", r["act"], inter, c["act"], hip.EPI_F32, r["y2"])
        after = seen[i + 1] if i + 1 < len(seen) else {"x": got, "xq": None}
        for j, (y, res, u, q, so) in enumerate([(r["y"], r["x"], r["mid"], r["midq"], c["mid"]),
                                                (r["y2"], r["mid"], after["x"], after["xq"], nxt)]):
            n64 = lambda t: t.cpu().numpy().astype(np.float64)  # noqa: E731
            _, _, ref_u = ref.residual_norm(n64(y), n64(res), None, 1.0, 0, None, None, 1, n64(layer.gamma[j]),
                                            n64(layer.beta[j]), enc.eps)
            assert np.abs(n64(u) - ref_u).max() <= 1e-5 * np.abs(ref_u).max()
            if q is not None:
                off = np.abs(rows(q, hidden) - np.clip(ref_u / float(f(so)), -127, 127))
                assert off.max() <= 0.5 + 2e-3, off.max()
    if not top_k:
        assert float((got - want).norm() / want.norm()) < 0.15
