"""The decoder of examples/decoder.py, prompts in one call and steps of one token: cache_append and both attentions of
every layer on what the operator before them left on the GPU, against the 64-bit definitions; the whole against the same
network in fp32; and a captured step, replayed, against eager ones.

Bars. Codes that cache_append stores: within half a step and 1e-3; attention's: within half a step, 4e-5 of 127 steps of
the values' scale and 1e-3 (test_gpu_cache.py derives both). Whole network: one int8 rounding is
under 1.4 % of an activation's root mean square (test_gpu_encoder_example.py); a layer has ten of them along its path, so
two layers stay under 30 % even if all of them add up.
"""
import os
import sys

import numpy as np
import pytest

import cache_ref as ref

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

LENS, STATES = [9, 1, 21, 5], [40, 77, 3, 16]


def build(hip):
    import torch
    from decoder import Decoder, batch_of
    dec = Decoder(layers=2, hidden=256, inter=512, heads=4, kv_heads=2, sparsity=0.7, page_size=16)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((sum(LENS), 256), device="cuda", generator=g)
    enc = torch.randn((sum(STATES), 256), device="cuda", generator=g)
    want = dec.calibrate(x, LENS, enc, STATES)
    start = batch_of(STATES)[0]
    states = dec.read(enc, start, torch.tensor(STATES, dtype=torch.int32, device="cuda"))
    return dec, x, want, states, batch_of


def check_layer(hip, dec, i, r, start, own, states, m):
    """One layer's append and attentions from what is on the device."""
    n = lambda t: t.cpu().numpy()  # noqa: E731
    f = lambda v: float(np.float32(v))  # noqa: E731
    c, nh, nkv, d = dec.scales[i], dec.heads, dec.kv_heads, dec.dim
    st, lens, table, cache = n(start), n(own.len), n(own.table), n(own.caches[i])
    queries, stored = ref.append(n(r["qkv"]).astype(np.float64), st, lens, table, 16, cache.shape[0], nh, nkv, d, ref.HALF,
                                 n(dec.inv_freq), 1.0)
    near = lambda code, v, s: np.abs(code - np.clip(v / f(s), -127, 127)).max()  # noqa: E731
    q = hip.from_t16x32(n(r["q"]), m, nh * d)
    for t, v in queries.items():
        assert near(q[t].reshape(nh, d), v, c["q"]) <= 0.5 + 1e-3
    for page, place, k, v in stored:
        for h in range(nkv):
            assert near(ref.key_of(cache, page, h, place), k[h], c["k"]) <= 0.5 + 1e-3
            assert near(ref.value_of(cache, page, h, place), v[h], c["v"]) <= 0.5 + 1e-3
    for name, q, at, scales, causal in (("att", "q", own, "qkv", True), ("catt", "cq", states, ("cq", "ck", "cv"), False)):
        q_scale, k_scale, v_scale = (f(c[s]) for s in scales)
        got = hip.from_t16x32(n(r[name]), m, nh * d)
        want, _ = ref.attention(hip.from_t16x32(n(r[q]), m, nh * d), n(at.caches[i]), st, n(at.len), n(at.table), nh,
                                q_scale * k_scale * f(d ** -0.5), causal)
        for t, v in want.items():
            bar = 0.5 + 4e-5 * 127 * v_scale / f(c[name]) + 1e-3
            assert near(got[t], v.reshape(-1) * v_scale, c[name]) <= bar, (name, t)


def test_prompt_then_steps(hip):
    import torch
    dec, x, want, states, batch_of = build(hip)
    own = dec.pages(len(LENS), max(LENS) + 4)
    start, longest = batch_of(LENS)
    own.len.copy_(torch.tensor(LENS, dtype=torch.int32))
    seen = []
    got = dec(x, start, longest, own, states, tap=lambda i, r: seen.append(r))
    torch.cuda.synchronize()
    for i, r in enumerate(seen):
        check_layer(hip, dec, i, r, start, own, states, x.shape[0])
    assert float((got - want).norm() / want.norm()) < 0.3
    one = torch.arange(len(LENS) + 1, dtype=torch.int32, device="cuda")
    last = got[start[1:].long() - 1]
    for _ in range(2):
        own.len.add_(1)
        seen.clear()
        last = dec(last, one, 1, own, states, tap=lambda i, r: seen.append(r))
        torch.cuda.synchronize()
        for i, r in enumerate(seen):
            check_layer(hip, dec, i, r, one, own, states, len(LENS))


def test_tokens_in_pieces_are_the_whole(hip):
    """Prompts token by token against the same in one call: the sums round otherwise, so codes may differ by a step, and
    what follows with them; each way stays within the bar of the fp32 network."""
    import torch
    dec, x, want, states, batch_of = build(hip)
    own = dec.pages(len(LENS), max(LENS))
    own.len.zero_()
    first = np.concatenate([[0], np.cumsum(LENS)])
    got = torch.zeros_like(want)
    for t in range(max(LENS)):
        at = [int(f) + t for f, n in zip(first, LENS) if t < n]
        start = torch.tensor(np.concatenate([[0], np.cumsum([t < n for n in LENS])]), dtype=torch.int32, device="cuda")
        own.len.add_((start[1:] > start[:-1]).int())
        got[at] = dec(x[at].contiguous(), start, 1, own, states)
    torch.cuda.synchronize()
    assert float((got - want).norm() / want.norm()) < 0.3


def test_a_captured_step_is_the_eager_one(hip):
    """Replayed several times, with eager work between, lengths growing on the device."""
    import torch
    dec, x, _, states, batch_of = build(hip)
    start, longest = batch_of(LENS)
    one = torch.arange(len(LENS) + 1, dtype=torch.int32, device="cuda")
    first = torch.randn((len(LENS), 256), device="cuda", generator=torch.Generator(device="cuda").manual_seed(9))

    def prompt():
        own = dec.pages(len(LENS), max(LENS) + 8)
        own.len.copy_(torch.tensor(LENS, dtype=torch.int32))
        dec(x, start, longest, own, states)
        return own

    torch.manual_seed(3)
    own = prompt()
    last, want = first.clone(), []
    for _ in range(6):
        own.len.add_(1)
        last = dec(last, one, 1, own, states)
        want.append(last.clone())
    own2 = prompt()
    last2 = first.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        own2.len.add_(1)
        dec(last2, one, 1, own2, states)
        own2.len.sub_(1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        own2.len.add_(1)
        last2.copy_(dec(last2, one, 1, own2, states))
    for i in range(6):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(last2, want[i]), i
        dec(x, start, longest, prompt(), states)  # eager work between
    assert torch.equal(own2.len, own.len)
