"""GPU tests of residual_norm through the C ABI against its definition in 64
bits, at odd widths, every type, layout, gate and norm, and where rows cross the
kernels' shapes.

Bars. With u32 = 2^-24: a row's sum of n terms is taken over at most D = 90
serial additions (64 values of a lane, 6 shuffles, 16 waves), so a sum is off by
at most D u32 times the sum of magnitudes, and an element passes through about
10 further roundings. One norm then gives |du| <= (D + 10) u32 (max|in| rstd
|gamma| + |beta|), and the second norm takes the first's error through its own
rstd. An int8 code has to lie within half a step and that error of u / scale.
"""
import numpy as np
import pytest

import encoder_ref as ref

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
D = 100


def _bar(x, kind, gamma, beta, eps, err):
    """Error bar (per row) of norm_rows(x) where x itself is off by at most err (per row)."""
    big = np.abs(x).max(1, keepdims=True)
    if kind == 0:
        return err
    mean = x.mean(1, keepdims=True) if kind == 1 else 0.0
    rstd = 1 / np.sqrt(np.square(x - mean).mean(1, keepdims=True) + eps)
    g = 1.0 if gamma is None else np.abs(gamma).max()
    b = 0.0 if beta is None else np.abs(beta).max()
    dev = np.abs(x - mean).max(1, keepdims=True) * rstd  # (an error of x also moves rstd)
    return (D * U32 * big + 2 * err) * rstd * g * (1 + dev) + D * U32 * (dev * g + b)


def _run(hip, m, n, y8, r, post, gate, kind, keep, layouts, seed=0, offset=0, affine=True, rscale=0.8, eps=1e-6):
    import torch
    rng = np.random.default_rng([seed, m, n])
    yl, rl, ql = layouts
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731

    def f32(*shape):
        return rng.normal(0.1, 1.0, shape).astype(np.float32)

    def put(a):  # fp32 tensors `offset` elements into an allocation
        if not offset or a.dtype != np.float32:
            return dev(a)
        buf = torch.empty(a.size + offset, dtype=torch.float32, device="cuda")
        view = buf[offset:].view(a.shape)
        view.copy_(dev(a))
        return view

    def act(is8, layout, scale):
        if not is8:
            a = f32(m, n)
            return a.astype(np.float64), put(a)
        c = rng.integers(-127, 128, (m, n), dtype=np.int8)
        t = hip.to_t16x32(c, fill=99) if layout else c
        return c.astype(np.float64) * np.float64(np.float32(scale)), dev(t)

    y, yd = act(y8, yl, 0.02)
    rv, rd = (None, None) if r == "none" else act(r == "i8", rl, 0.03)
    gv = {"none": None, "channel": (n,), "token": (m, 1), "element": (m, n)}[gate]
    gv = None if gv is None else rng.uniform(-1, 1, gv).astype(np.float32)
    w = [f32(n) if affine else None for _ in range(4)]
    d64 = [None if a is None else a.astype(np.float64) for a in w]
    t, h, u = ref.residual_norm(y, rv, None if gv is None else gv.astype(np.float64), float(np.float32(rscale)), post,
                                d64[0], d64[1], kind, d64[2], d64[3], eps)
    so = float(np.float32(max(np.abs(u).max(), 1e-3) / 120))
    wd = [None if a is None else put(a) for a in w]
    got = hip.residual_norm(yd, wd[2], wd[3], norm=kind, eps=eps, y_scale=0.02, residual=rd, residual_scale=rscale,
                            r_scale=0.03, gate=None if gv is None else put(gv), post_norm=post, post_gamma=wd[0],
                            post_beta=wd[1], keep_sum="h" in keep, keep_norm="u" in keep,
                            out_scale=so if "q" in keep else None, y_layout=yl, r_layout=rl, q_layout=ql, shape=(m, n))
    torch.cuda.synchronize()
    err_t = _bar(y, post, d64[0], d64[1], eps, 0.0)
    size = np.abs(t).max(1, keepdims=True) + (0 if rv is None else np.abs(rv).max(1, keepdims=True))
    err_h = err_t + 8 * U32 * size
    err_u = _bar(h, kind, d64[2], d64[3], eps, err_h) + 8 * U32 * np.abs(u).max(1, keepdims=True)
    for name, out, want, err in (("h", got[0], h, err_h), ("u", got[1], u, err_u)):
        assert (out is not None) == (name in keep)
        if out is not None:
            bad = np.abs(out.cpu().numpy() - want) - err
            assert bad.max() <= 0, f"{name}: {bad.max()} over the bar"
    assert (got[2] is not None) == ("q" in keep)
    if got[2] is not None:
        q = got[2].cpu().numpy()
        q = hip.from_t16x32(q, m, n) if ql else q
        z = np.clip(u / so, -127, 127)
        off = np.abs(q - z) - (0.5 + err_u / so + 4 * U32 * 128)
        assert off.max() <= 0 and q.min() >= -127, f"codes: {off.max()} over the bar"


WIDTHS = [1, 2, 3, 4, 5, 31, 33, 256, 257, 511, 768, 1000, 1001, 1024, 1028, 2048, 2052, 4096, 4100, 16384, 16388, 65535]


@pytest.mark.parametrize("n", WIDTHS)
def test_widths(hip, n):
    for i, m in enumerate((1, 5, 19)):
        _run(hip, m, n, i == 1, ("f32", "i8", "none")[i], (0, 1, 2)[i], ("none", "channel", "element")[i],
             (1, 2, 1)[i], "huq", ((0, 0, 0), (1, 1, 1), (0, 0, 1))[i], seed=i)


@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "element"])
def test_norms_and_gates(hip, post, kind, gate):
    for r in ("none", "f32", "i8"):
        for y8 in (False, True):
            _run(hip, 37, 200, y8, r, post, gate, kind, "huq", (1, 0, 1), seed=kind)


@pytest.mark.parametrize("layouts", [(0, 0, 0), (0, 0, 1), (1, 0, 0), (0, 1, 1), (1, 1, 1)])
@pytest.mark.parametrize("keep", ["q", "h", "u", "hu", "uq"])
def test_layouts_and_outputs(hip, layouts, keep):
    for n in (70, 96):
        _run(hip, 33, n, True, "i8", 1, "none", 1, keep, layouts)


@pytest.mark.parametrize("offset", [1, 2, 4])
def test_alignment(hip, offset):
    for n in (64, 768, 4096):
        _run(hip, 9, n, False, "f32", 2, "channel", 1, "huq", (0, 0, 0), offset=offset)


def test_no_affine_and_zero_rows(hip):
    import torch
    _run(hip, 20, 300, False, "f32", 1, "none", 2, "huq", (0, 0, 0), affine=False)
    z = torch.zeros((4, 64), device="cuda")
    h, u, q = hip.residual_norm(z, eps=1e-5, residual=z, keep_sum=True, keep_norm=True, out_scale=0.1)
    for t in (h, u, q):
        assert int((t != 0).sum()) == 0  # a constant row is no reason for NaN
    e = hip.residual_norm(torch.empty((0, 64), device="cuda"), keep_sum=True, out_scale=0.1)
    assert e[0].shape == (0, 64) and e[2].shape == (0, 64)


def test_large_means(hip):
    """A mean a thousand times the spread: the squared deviations are taken from the mean, not from zero."""
    import torch
    rng = np.random.default_rng(3)
    x = (1000 + rng.normal(0, 1, (8, 768))).astype(np.float32)
    x64 = x.astype(np.float64)
    _, u, _ = hip.residual_norm(torch.from_numpy(x).cuda(), eps=1e-6, keep_norm=True)
    want = ref.norm_rows(x64, 1, None, None, 1e-6)
    assert np.abs(u.cpu().numpy() - want).max() <= _bar(x64, 1, None, None, 1e-6, 0.0).max()


def test_not_a_number_stays_in_its_row(hip):
    import torch
    x = torch.randn((40, 768), device="cuda")
    clean = hip.residual_norm(x, keep_sum=True, keep_norm=True)
    x[7, 5], x[20, 0] = float("nan"), float("inf")
    got = hip.residual_norm(x, keep_sum=True, keep_norm=True)
    keep = torch.ones(40, dtype=torch.bool)
    keep[7] = keep[20] = False
    for a, b in zip(got[:2], clean[:2]):
        assert torch.equal(a.cpu()[keep], b.cpu()[keep])
        assert torch.isnan(got[1].cpu()[~keep]).any(1).all()


def test_in_place(hip):
    import torch
    for n in (768, 4096, 1001):
        y, r = torch.randn((33, n), device="cuda"), torch.randn((33, n), device="cuda")
        h, u, _ = hip.residual_norm(y, residual=r, keep_sum=True, keep_norm=True)
        y2, r2 = y.clone(), r.clone()
        h2, u2, _ = hip.residual_norm(y2, residual=r2, keep_sum=r2, keep_norm=y2)
        assert h2 is r2 and u2 is y2 and torch.equal(h2, h) and torch.equal(u2, u)


def test_graph_and_stream(hip):
    """Captured once and replayed, on a stream of its own, with eager work between the replays."""
    import torch
    y, r = torch.randn((300, 768), device="cuda"), torch.randn((300, 768), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(y), torch.empty_like(y), torch.empty(y.shape, dtype=torch.int8, device="cuda")

    def step():
        hip.residual_norm(y, residual=r, keep_sum=out[0], keep_norm=out[1], out_scale=0.03, q_out=out[2])

    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        y.normal_()
        r.mul_(0.5 + i)
        graph.replay()
        torch.cuda.synchronize()
        want = hip.residual_norm(y, residual=r, keep_sum=True, keep_norm=True, out_scale=0.03)
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("n", [513, 600, 768, 769, 1001, 1024])
def test_widths_of_many_rows(hip, n):
    """More rows than a row is given four waves for, and the last of those."""
    for i, m in enumerate((2048, 2049, 2103)):
        _run(hip, m, n, i == 1, ("f32", "i8", "none")[i], (0, 1, 2)[i], ("none", "channel", "element")[i],
             (1, 2, 1)[i], "huq", ((0, 0, 0), (1, 1, 1), (0, 0, 1))[i], seed=i)


@pytest.mark.parametrize("n", [2049, 2560, 3013, 3071, 3073, 3999, 4095])
def test_widths_between_2048_and_4096(hip, n):
    for i, m in enumerate((1, 6, 19)):
        _run(hip, m, n, i == 1, ("f32", "i8", "none")[i], (0, 1, 2)[i], ("none", "channel", "element")[i],
             (1, 2, 1)[i], "huq", ((0, 0, 0), (1, 1, 1), (0, 0, 1))[i], seed=i)
