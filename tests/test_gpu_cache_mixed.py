"""One prompt beside many steps in a call of a decoder's cache: so many sequences that there is no workgroup for each of
the prompt's tiles times the sequences, against the definition in 64 bits. The bar is test_gpu_cache.py's."""
import pytest

from test_gpu_cache import FILL, TOL

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
