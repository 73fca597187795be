"""A DistilBERT-shaped encoder on this library, int8 activations end to end:

    QKV -> attention -> attention output -> LayerNorm(x + .) -> FFN1 -> FFN2 -> LayerNorm(x + .)

    python examples/encoder.py [--layers 6] [--batch 32] [--seq 128] [--sparsity 0.8] [--top-k K]

Weights are random 4x1-block-sparse ones. Sequences of a batch lie one after the
other without padding; --ragged draws their lengths. With --top-k every block of
64 queries attends to that many blocks of 64 keys, chosen by pooled scores (for
long documents). Scales are calibrated by largest magnitude on the same network
in fp32, which the output is then compared with.
"""
import argparse
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2211_07715_amd as sl  # noqa: E402
from workloads import make_weight  # noqa: E402

BLOCKS = sl.LAYOUT_T16X32
LINEARS = ("qkv", "out", "ffn1", "ffn2")


class Layer:
    """Weights of one layer, dense on the host and packed on the device, and its two norms."""

    def __init__(self, hidden, inter, sparsity, seed):
        self.dense, self.packed = {}, {}
        shapes = {"qkv": (3 * hidden, hidden), "out": (hidden, hidden), "ffn1": (inter, hidden), "ffn2": (hidden, inter)}
        for op, (name, (n, k)) in enumerate(shapes.items()):
            d = make_weight(n, k, sparsity, seed=seed, op=op)
            d["sw"] = np.full(n, 1.5 / (73 * math.sqrt(k * (1 - sparsity))), np.float32)  # outputs of about x's size
            self.dense[name] = d
            self.packed[name] = sl.PackedWeight.pack(d["w"], d["sw"], d["b"])
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.gamma = [1 + 0.1 * torch.randn(hidden, device="cuda", generator=g) for _ in range(2)]
        self.beta = [0.05 * torch.randn(hidden, device="cuda", generator=g) for _ in range(2)]

    def plain(self, name, x):
        d = self.dense[name]
        w = torch.from_numpy(d["w"]).cuda().float() * torch.from_numpy(d["sw"]).cuda()[:, None]
        return x @ w.t() + torch.from_numpy(d["b"]).cuda()


class Encoder:
    def __init__(self, layers=6, hidden=768, inter=3072, heads=12, sparsity=0.8, seed=0, eps=1e-12):
        self.hidden, self.heads, self.eps = hidden, heads, eps
        self.layers = [Layer(hidden, inter, sparsity, seed + i) for i in range(layers)]
        self.scales = None

    def calibrate(self, x, lens, top_k=0):
        """fp32 forward of the same network; sets every activation's scale from its largest magnitude."""
        self.scales = []
        for layer in self.layers:
            s = {"x": x}
            s["qkv"] = layer.plain("qkv", x)
            s["att"] = self._plain_attention(s["qkv"], lens, top_k)
            norm = lambda v, i: torch.nn.functional.layer_norm(  # noqa: E731
                v, (self.hidden,), layer.gamma[i], layer.beta[i], self.eps)
            s["mid"] = norm(x + layer.plain("out", s["att"]), 0)
            s["act"] = torch.nn.functional.gelu(layer.plain("ffn1", s["mid"]))
            x = norm(s["mid"] + layer.plain("ffn2", s["act"]), 1)
            self.scales.append({k: float(v.abs().max()) / 127 for k, v in s.items()})
        self.scales.append({"x": float(x.abs().max()) / 127})
        return x

    def _plain_attention(self, qkv, lens, top_k):
        d = self.hidden // self.heads
        out, first = [], 0
        for n in lens:
            q, k, v = qkv[first:first + n].reshape(n, 3, self.heads, d).permute(1, 2, 0, 3).contiguous()
            z = q @ k.transpose(1, 2).contiguous() / math.sqrt(d)
            if top_k and -(-n // 64) > top_k:  # the blocks of largest pooled score, for each block of 64 queries
                pool = lambda t: torch.stack([c.mean(1) for c in t.split(64, dim=1)], 1)  # noqa: E731
                score = pool(q) @ pool(k).transpose(1, 2).contiguous()
                use = torch.zeros_like(score, dtype=torch.bool).scatter_(2, score.topk(top_k, dim=2).indices, True)
                at = torch.arange(n, device=z.device) // 64
                z = z.masked_fill(~use[:, at][:, :, at], -math.inf)
            out.append((torch.softmax(z, 2) @ v).transpose(0, 1).reshape(n, self.hidden))
            first += n
        return torch.cat(out)

    def __call__(self, x, start, longest, top_k=0, tap=None):
        """x: fp32 [tokens, hidden]; start: int32 sequence starts on the device. tap(i, results) sees
        what layer i left on the device, by name."""
        m, d, s = x.shape[0], self.hidden // self.heads, self.scales
        tap = tap or (lambda *a: None)
        blocks = dict(x_layout=BLOCKS, m_tokens=m)
        xq = sl.quantize_act(x, s[0]["x"], layout=BLOCKS)
        for i, layer in enumerate(self.layers):
            run, c = layer.packed, s[i]
            qkv = run["qkv"].run(xq, c["x"], sl.EPI_I8, out_scale=c["qkv"], y_layout=BLOCKS, **blocks)
            lists = sl.select_blocks(qkv, start, longest, self.heads, d, top_k, **blocks) if top_k else None
            att = sl.attention(qkv, c["qkv"], start, longest, self.heads, d, out_scale=c["att"], blocks=lists,
                               y_layout=BLOCKS, **blocks)
            y = run["out"].run(att, c["att"], sl.EPI_F32, **blocks)
            _, mid, midq = sl.residual_norm(y, layer.gamma[0], layer.beta[0], eps=self.eps, residual=x, keep_norm=True,
                                            out_scale=c["mid"], q_layout=BLOCKS)
            act = run["ffn1"].run(midq, c["mid"], sl.EPI_I8_GELU, out_scale=c["act"], y_layout=BLOCKS, **blocks)
            y2 = run["ffn2"].run(act, c["act"], sl.EPI_F32, **blocks)
            tap(i, dict(x=x, xq=xq, qkv=qkv, lists=lists, att=att, y=y, mid=mid, midq=midq, act=act, y2=y2))
            _, x, xq = sl.residual_norm(y2, layer.gamma[1], layer.beta[1], eps=self.eps, residual=mid, keep_norm=True,
                                        out_scale=s[i + 1]["x"], q_layout=BLOCKS)
        return x


def batch_of(lens):
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return torch.from_numpy(start).cuda(), int(max(lens))


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, kind, value in (("layers", int, 6), ("batch", int, 32), ("seq", int, 128), ("sparsity", float, 0.8),
                              ("top-k", int, 0), ("steps", int, 20)):
        p.add_argument("--" + name, type=kind, default=value)
    p.add_argument("--ragged", action="store_true")
    a = p.parse_args()
    rng = np.random.default_rng(0)
    lens = rng.integers(1, a.seq + 1, a.batch).tolist() if a.ragged else [a.seq] * a.batch
    start, longest = batch_of(lens)
    x = torch.randn((sum(lens), 768), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    enc = Encoder(layers=a.layers, sparsity=a.sparsity)
    want = enc.calibrate(x, lens, a.top_k)
    got = enc(x, start, longest, a.top_k)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        enc(x, start, longest, a.top_k)
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / a.steps
    err = float((got - want).norm() / want.norm())
    print(f"{len(lens)} sequences, {sum(lens)} tokens, {a.layers} layers: {t * 1e6:.0f} us ({t * 1e6 / a.layers:.0f} a "
          f"layer, host launches included), {sum(lens) / t:.0f} tokens/s; against fp32: {100 * err:.1f} %")


if __name__ == "__main__":
    main()
