"""A decoder beside the encoder of encoder.py, int8 activations end to end: rotated
self-attention over a paged cache, attention to an encoder's states, feed-forward.

    QKV -> append, attention -> output -> LayerNorm(x + .) ->
    Q -> attention to the states -> output -> LayerNorm(x + .) -> FFN1 -> FFN2 -> LayerNorm(x + .)

    python examples/decoder.py [--layers 6] [--batch 32] [--prompt 16] [--states 128] [--steps 64]

Weights are random 4x1-block-sparse ones, key and value heads are shared by pairs of
query heads. Prompts go in one call, then every step adds one token a sequence: its
input here is the output of the step before, and the step, whose lengths live on
the device, is captured into a graph and replayed. Scales are calibrated by largest
magnitude on the same network in fp32.
"""
import argparse
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2211_07715_amd as sl  # noqa: E402
from encoder import Layer, batch_of  # noqa: E402

BLOCKS = sl.LAYOUT_T16X32


def linears(hidden, inter, kv):
    return {"qkv": (hidden + 2 * kv, hidden), "out": (hidden, hidden), "cq": (hidden, hidden), "ckv": (2 * kv, hidden),
            "cout": (hidden, hidden), "ffn1": (inter, hidden), "ffn2": (hidden, inter)}


class Pages:
    """A cache for each layer and the page tables of a batch; sequence s takes its pages as it needs them."""

    def __init__(self, layers, batch, longest, kv_heads, head_dim, page_size):
        per = -(-longest // page_size)
        shape = sl.cache_shape(batch * per, page_size, kv_heads, head_dim)
        self.caches = [torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(layers)]
        self.table = torch.randperm(batch * per, device="cuda").to(torch.int32).reshape(batch, per)
        self.len = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.longest = longest


class Decoder:
    def __init__(self, layers=6, hidden=768, inter=None, heads=12, kv_heads=6, sparsity=0.8, seed=0, eps=1e-12,
                 page_size=64):
        self.hidden, self.heads, self.kv_heads, self.eps, self.page_size = hidden, heads, kv_heads, eps, page_size
        self.dim = hidden // heads
        self.layers = [Layer(hidden, inter, sparsity, seed + i, linears(hidden, inter or 4 * hidden, kv_heads * self.dim), norms=3)
                       for i in range(layers)]
        self.inv_freq = (10000.0 ** (-torch.arange(0, self.dim, 2, dtype=torch.float64) / self.dim)).float().cuda()
        self.scales = None

    def pages(self, batch, longest):
        return Pages(len(self.layers), batch, longest, self.kv_heads, self.dim, self.page_size)

    # --- fp32 ---------------------------------------------------------------

    def _rotate(self, x, pos):
        w = (pos.double()[:, None, None] * self.inv_freq.double())
        c, s, (a, b) = w.cos().float(), w.sin().float(), x.chunk(2, 2)
        return torch.cat([a * c - b * s, b * c + a * s], 2)

    def _plain_attention(self, q, k, v, causal):
        g = self.heads // self.kv_heads
        q, k, v = (t.transpose(0, 1) for t in (q, k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)))
        z = q @ k.transpose(1, 2).contiguous() / math.sqrt(self.dim)
        if causal:
            z = z.masked_fill(torch.ones(z.shape[1:], dtype=torch.bool, device=z.device).triu(1), -math.inf)
        return (torch.softmax(z, 2) @ v.contiguous()).transpose(0, 1).reshape(-1, self.hidden)

    def calibrate(self, x, lens, states, state_lens):
        """fp32 forward over whole sequences; sets every activation's scale from its largest magnitude."""
        split = lambda t, heads: t.reshape(t.shape[0], heads, self.dim)  # noqa: E731
        nh, nkv = self.heads, self.kv_heads
        pos = torch.cat([torch.arange(n, device=x.device) for n in lens])
        self.scales = []
        for layer in self.layers:
            s = {"x": x, "states": states}
            norm = lambda v, i: torch.nn.functional.layer_norm(  # noqa: E731
                v, (self.hidden,), layer.gamma[i], layer.beta[i], self.eps)
            qkv = split(layer.plain("qkv", x), nh + 2 * nkv)
            qk, v = self._rotate(qkv[:, :nh + nkv], pos), qkv[:, nh + nkv:]
            s["q"], s["k"], s["v"] = qk[:, :nh], qk[:, nh:], v
            parts = zip(*(t.split(lens) for t in (s["q"], s["k"], v)))
            s["att"] = torch.cat([self._plain_attention(*t, True) for t in parts])
            s["mid"] = norm(x + layer.plain("out", s["att"]), 0)
            s["cq"] = split(layer.plain("cq", s["mid"]), nh)
            ckv = split(layer.plain("ckv", states), 2 * nkv)
            s["ck"], s["cv"] = ckv[:, :nkv], ckv[:, nkv:]
            parts = zip(s["cq"].split(lens), s["ck"].split(state_lens), s["cv"].split(state_lens))
            s["catt"] = torch.cat([self._plain_attention(*t, False) for t in parts])
            s["mid2"] = norm(s["mid"] + layer.plain("cout", s["catt"]), 1)
            s["act"] = torch.nn.functional.gelu(layer.plain("ffn1", s["mid2"]))
            x = norm(s["mid2"] + layer.plain("ffn2", s["act"]), 2)
            self.scales.append({k: float(t.abs().max()) / 127 for k, t in s.items()})
        self.scales.append({"x": float(x.abs().max()) / 127})
        return x

    # --- int8 ---------------------------------------------------------------

    def read(self, states, start, lens):
        """Keys and values of an encoder's states (fp32 [tokens, hidden]), once for all steps: a cache of their own."""
        pages, m = self.pages(lens.shape[0], int(lens.max())), states.shape[0]
        pages.len.copy_(lens)
        for layer, c, cache in zip(self.layers, self.scales, pages.caches):
            xq = sl.quantize_act(states, c["states"], layout=BLOCKS)
            kv = layer.packed["ckv"].run(xq, c["states"], sl.EPI_F32, m_tokens=m, x_layout=BLOCKS)
            sl.cache_append(kv, cache, pages.table, start, pages.len, pages.longest, 0, k_scale=c["ck"], v_scale=c["cv"])
        return pages

    def __call__(self, x, start, most_new, own, states, tap=None):
        """The sequences' next tokens: fp32 [tokens, hidden], sequence starts on the device, at most most_new each;
        own.len counts them already. tap(i, results) sees what layer i left on the device, by name."""
        m, nh = x.shape[0], self.heads
        tap = tap or (lambda *a: None)
        blocks = dict(x_layout=BLOCKS, m_tokens=m)
        xq = sl.quantize_act(x, self.scales[0]["x"], layout=BLOCKS)
        for i, layer in enumerate(self.layers):
            run, c, nxt = layer.packed, self.scales[i], self.scales[i + 1]["x"]

            def norm(y, residual, j, scale):
                return sl.residual_norm(y, layer.gamma[j], layer.beta[j], eps=self.eps, residual=residual, keep_norm=True,
                                        out_scale=scale, q_layout=BLOCKS)[1:]

            def attend(q, cache, at, scales, causal):
                sq, sk, sv, so = (c[k] for k in scales)
                return sl.cache_attention(q, cache, at.table, start, at.len, most_new, at.longest, nh, q_scale=sq,
                                          k_scale=sk, v_scale=sv, causal=causal, out_scale=so, q_layout=BLOCKS,
                                          y_layout=BLOCKS, m_tokens=m)

            qkv = run["qkv"].run(xq, c["x"], sl.EPI_F32, **blocks)
            q = sl.cache_append(qkv, own.caches[i], own.table, start, own.len, most_new, nh, q_scale=c["q"],
                                k_scale=c["k"], v_scale=c["v"], rope=sl.ROPE_HALF, inv_freq=self.inv_freq, q_layout=BLOCKS)
            att = attend(q, own.caches[i], own, ("q", "k", "v", "att"), True)
            mid, midq = norm(run["out"].run(att, c["att"], sl.EPI_F32, **blocks), x, 0, c["mid"])
            cq = run["cq"].run(midq, c["mid"], sl.EPI_I8, out_scale=c["cq"], y_layout=BLOCKS, **blocks)
            catt = attend(cq, states.caches[i], states, ("cq", "ck", "cv", "catt"), False)
            mid2, mid2q = norm(run["cout"].run(catt, c["catt"], sl.EPI_F32, **blocks), mid, 1, c["mid2"])
            act = run["ffn1"].run(mid2q, c["mid2"], sl.EPI_I8_GELU, out_scale=c["act"], y_layout=BLOCKS, **blocks)
            tap(i, dict(qkv=qkv, q=q, att=att, cq=cq, catt=catt))
            x, xq = norm(run["ffn2"].run(act, c["act"], sl.EPI_F32, **blocks), mid2, 2, nxt)
        return x


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("layers", 6), ("batch", 32), ("prompt", 16), ("states", 128), ("steps", 64)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    dec = Decoder(layers=a.layers)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, enc = (torch.randn((a.batch * n, dec.hidden), device="cuda", generator=g) for n in (a.prompt, a.states))
    dec.calibrate(x, [a.prompt] * a.batch, enc, [a.states] * a.batch)
    states = dec.read(enc, *[batch_of([a.states] * a.batch)[0], torch.full((a.batch,), a.states, device="cuda")])
    own = dec.pages(a.batch, a.prompt + a.steps)
    own.len.fill_(a.prompt)
    last = dec(x, batch_of([a.prompt] * a.batch)[0], a.prompt, own, states)[a.prompt - 1::a.prompt].clone()
    one = torch.arange(a.batch + 1, dtype=torch.int32, device="cuda")
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):  # (its token is written again by the first step)
        own.len.add_(1)
        dec(last, one, 1, own, states)
        own.len.sub_(1)
    torch.cuda.current_stream().wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        own.len.add_(1)
        last.copy_(dec(last, one, 1, own, states))
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / a.steps
    print(f"{a.batch} sequences, {a.prompt} + {a.steps} tokens each over {a.states} states, {a.layers} layers: "
          f"{t * 1e6:.0f} us a step ({t * 1e6 / a.layers:.0f} a layer), {a.batch / t:.0f} tokens/s")


if __name__ == "__main__":
    main()
