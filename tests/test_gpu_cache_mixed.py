"""One prompt beside many steps in a call of a decoder's cache: so many sequences that there is no workgroup for each of
the prompt's tiles (or groups of 16 slots) times the sequences, against the definitions in 64 bits. The bars are
test_gpu_cache.py's."""
import pytest

from test_gpu_cache import DELTA, FILL, TOL

pytestmark = pytest.mark.gpu

PS = 16
# sequences, the prompt's place among them, its tokens, query and key heads, features of a head
MIXED = [(60001, 31007, 1000, 32, 8, 16), (256, 100, 4224, 1000, 1000, 16)]


class Mixed:
    """Sequences of one token with 0 to 3 cached ones, each in a page of its own, and one prompt."""

    def __init__(self, hip, n, at, prompt, nkv, hd):
        import torch
        self.n, self.at, self.prompt, self.nkv, self.hd = n, at, prompt, nkv, hd
        self.gen = g = torch.Generator(device="cuda").manual_seed(n)
        per = -(-prompt // PS)
        pages = torch.randperm(n - 1 + per, device="cuda", generator=g).to(torch.int32)
        self.table = torch.full((n, per), -1, dtype=torch.int32, device="cuda")
        self.steps = torch.arange(n, device="cuda") != at
        self.table[self.steps, 0] = pages[:n - 1]
        self.table[at] = pages[n - 1:]
        news = torch.where(self.steps, 1, prompt)
        self.m = int(news.sum())
        self.start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), news.cumsum(0)]).to(torch.int32)
        self.len = torch.randint(0, 4, (n,), device="cuda", generator=g, dtype=torch.int32)
        self.len[at] = prompt
        self.cache = self.codes(*hip.cache_shape(n - 1 + per, PS, nkv, hd))
        self.first = self.start[self.steps.nonzero()[:, 0]].long()  # the steps' tokens
        self.rows = slice(at, at + prompt)                          # and the prompt's

    def codes(self, *shape):
        import torch
        return torch.randint(-127, 128, shape, device="cuda", generator=self.gen, dtype=torch.int8)

    def call(self):
        return self.cache, self.table, self.start, self.len, self.prompt

    def keys_and_values(self, pages, h):
        """[.., PS, hd] of one head, in 64 bits."""
        v = self.cache[pages, 1, h].reshape(*pages.shape, 1, self.hd, PS)[..., 0, :, :].transpose(-1, -2)
        return self.cache[pages, 0, h].double(), v.double().contiguous()


@pytest.mark.parametrize("n,at,prompt,nh,nkv,hd", MIXED)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(hip, n, at, prompt, nh, nkv, hd, causal):
    import numpy as np
    import torch
    b = Mixed(hip, n, at, prompt, nkv, hd)
    q = b.codes(b.m, nh * hd)
    f = lambda v: float(np.float32(v))  # noqa: E731
    qs, ks, vs, g = 0.02, 0.03, 0.03, nh // nkv
    y = torch.full((b.m, nh * hd), float(FILL), device="cuda")
    print(f"attention of a prompt beside steps: {n} sequences, {prompt} tokens, causal={causal}", flush=True)
    hip.cache_attention(q, *b.call(), prompt, nh, q_scale=qs, k_scale=ks, v_scale=vs, causal=causal, kind=hip.EPI_F32, out=y)
    torch.cuda.synchronize()
    assert hip.last_path() == f"cache prompt {hd},1"
    scale = f(qs) * f(ks) * f(hd ** -0.5)
    own = b.table[b.steps, 0].long()
    unseen = torch.arange(PS, device="cuda")[None, None] >= b.len[b.steps].long()[:, None, None]
    later = torch.ones((prompt, prompt), dtype=torch.bool, device="cuda").triu(1) if causal else None
    worst = 0.0
    for h in range(nkv):
        heads = slice(h * g * hd, (h + 1) * g * hd)
        k, v = b.keys_and_values(own, h)
        z = (q[b.first, heads].reshape(-1, g, hd).double() @ k.transpose(1, 2).contiguous() * scale)
        w = torch.softmax(z.masked_fill(unseen, -torch.inf), 2).nan_to_num(0.0)  # (nothing seen: 0)
        worst = max(worst, float((y[b.first, heads].reshape(-1, g, hd) - w @ v * f(vs)).abs().max()))
        k, v = (t.reshape(-1, hd)[:prompt] for t in b.keys_and_values(b.table[at].long(), h))
        for a in range(h * g, (h + 1) * g):
            head = slice(a * hd, (a + 1) * hd)
            z = q[b.rows, head].double() @ k.t().contiguous() * scale
            if causal:
                z.masked_fill_(later, -torch.inf)
            worst = max(worst, float((y[b.rows, head] - torch.softmax(z, 1) @ v * f(vs)).abs().max()))
    assert worst <= TOL * vs, worst


@pytest.mark.parametrize("x_type", ["i8", "f32"])
def test_append(hip, x_type):
    import numpy as np
    import torch
    n, at, prompt, nh, nkv, hd = MIXED[0]
    b = Mixed(hip, n, at, prompt, nkv, hd)
    b.len[at] = prompt - 5  # (its first five tokens have no slot)
    f = lambda v: float(np.float32(v))  # noqa: E731
    xs, qs, ks, vs = 0.031, 0.037, 0.041, 0.031
    x = b.codes(b.m, (nh + 2 * nkv) * hd)
    value = (x.double() * f(xs)).reshape(b.m, nh + 2 * nkv, hd)
    if x_type == "f32":
        x = value.reshape(b.m, -1).float()
        value = x.double().reshape(value.shape)
    freq = torch.tensor(10000.0 ** (-np.arange(hd // 2) * 2 / hd), dtype=torch.float32, device="cuda")
    before = b.cache.clone()
    print(f"append of a prompt beside steps: {n} sequences, {prompt} tokens, {x_type}", flush=True)
    q = hip.cache_append(x, *b.call(), nh, x_scale=xs if x_type == "i8" else 1.0, q_scale=qs, k_scale=ks, v_scale=vs,
                         rope=hip.ROPE_HALF, inv_freq=freq)
    torch.cuda.synchronize()
    # every token's sequence, slot and page
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), torch.where(b.steps, 1, prompt))
    start, lens = b.start.long(), b.len.long()
    slot = lens[seq] - (start[seq + 1] - start[seq]) + torch.arange(b.m, device="cuda") - start[seq]
    w = slot.double()[:, None] * freq.double()
    c, s, (u, v) = w.cos()[:, None], w.sin()[:, None], value[:, :nh + nkv].chunk(2, 2)
    turned = torch.cat([u * c - v * s, v * c + u * s], 2)

    def near(codes, want, scale):
        want = (want / f(scale)).clamp(-127, 127)
        assert float((codes.double() - want).abs().max()) <= 0.5 + DELTA

    near(q.reshape(b.m, nh, hd), turned[:, :nh], qs)
    put = slot >= 0
    page, place = b.table[seq[put], slot[put] // PS].long(), slot[put] % PS
    assert int((~put).sum()) >= 5 and int(page.min()) >= 0
    near(b.cache[page, 0, :, place], turned[put, nh:], ks)
    got, was = (t[:, 1].reshape(-1, nkv, hd, PS) for t in (b.cache, before))
    near(got[page, :, :, place], value[put, nh + nkv:], vs)
    # what no token of the call is in stays as it was
    before[page, 0, :, place] = b.cache[page, 0, :, place]
    was[page, :, :, place] = got[page, :, :, place]
    assert torch.equal(b.cache[:, 0], before[:, 0]) and torch.equal(got, was)
