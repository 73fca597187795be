"""What the speed of the operators between the sparse linears is measured on:
``residual_norm``, ``attention`` and ``select_blocks``, as a serving program of an
int8 encoder calls them.

``own`` false: every operator in its plain form, elementary torch operations in
32 bits. ``own`` true: the calls of this package. A case is a dict of plain
values; ``op`` says what one pass is:

    norm       one ``residual_norm``: an optional norm of a block's output, its
               gate, the scaled residual, the next block's norm, and the int8
               codes that the next linear reads
    attention  the attention core on the int8 output of a fused QKV linear
    select     the choice of key blocks for every query block and head
    blocks     that choice, and the attention over the chosen blocks

Sequences of a batch lie one after the other, without padding between them
(``lens``: ``b`` sequences of ``s`` tokens, ``ragged``: lengths drawn from 1 to
``s``); with ``masked`` each also has its own number of valid keys, zero for
one of them. Activations are int8 codes, normal by token with a slowly changing
part (neighbouring tokens resemble each other); ``layout`` is that of the int8
activations: ``rows`` or ``tiles`` (16 tokens x 32 features). Int8 results are
returned as the values they stand for, in bfloat16.
"""
import math

import torch

own = False

BLOCK = 64    # keys of a selectable block
ROWS, TILES = 0, 1  # the package's numbers of the two layouts
F32, I8 = 1, 3      # and of its fp32 and int8 results
LAYER, RMS = 1, 2   # and of its norms
EPS = 1e-12


def _norm(name, m, n, y, r, post, gate, norm, rscale, keep, layout):
    return dict(name=name, op="norm", m=m, n=n, y=y, r=r, post=post, gate=gate, norm=norm, rscale=rscale, keep=keep,
                layout=layout)


def _att(name, op, b, s, ragged, masked, nh, nkv, hd, kind, layout, top_k=0, qb=0):
    return dict(name=name, op=op, b=b, s=s, ragged=ragged, masked=masked, nh=nh, nkv=nkv, hd=hd, kind=kind,
                layout=layout, top_k=top_k, qb=qb)


def listed():
    return [
        # the smallest: after the attention output of one short sequence
        _norm("norm_b1_s128", 128, 768, "i8", "f32", "none", "none", "layer", 1.0, "u", "tiles"),
        # after FFN2 (fp32) of a DistilBERT layer at batch 32: sum, LayerNorm, codes for the next QKV
        _norm("norm_b32_s128", 4096, 768, "f32", "f32", "none", "none", "layer", 1.0, "u", "tiles"),
        # odd sizes: unpadded sequences, a width that is no multiple of 4, norms on both sides, a gate for each element
        _norm("norm_ragged", 1531, 1001, "f32", "f32", "rms", "element", "rms", 0.8, "h", "rows"),
        # throughput serving of long sequences, norms on both sides and a gate for each channel
        _norm("norm_b128_s384", 49152, 1024, "i8", "f32", "layer", "channel", "layer", 1.0, "h", "tiles"),
        # batch-1 latency of the attention core
        _att("attn_b1_s128", "attention", 1, 128, False, False, 12, 12, 64, "i8", "rows"),
        # a DistilBERT layer at batch 32
        _att("attn_b32_s128", "attention", 32, 128, False, False, 12, 12, 64, "i8", "tiles"),
        # unpadded sequences of 1 to 384 tokens with masked keys, fp32 results
        _att("attn_ragged", "attention", 24, 384, True, True, 12, 12, 64, "f32", "rows"),
        # throughput serving
        _att("attn_b128_s384", "attention", 128, 384, False, False, 12, 12, 64, "i8", "tiles"),
        # a long document, key and value heads shared by 4 query heads
        _att("attn_s8192", "attention", 1, 8192, False, False, 16, 4, 64, "i8", "rows"),
        # the choice alone
        _att("select_b2_s4096", "select", 2, 4096, False, False, 12, 12, 64, "i8", "tiles", 16, 64),
        # a very long document over an eighth of its blocks
        _att("blocks_s16384", "blocks", 1, 16384, False, False, 12, 12, 64, "i8", "tiles", 32, 64),
        # long documents of odd lengths, wide heads, a coarser choice, fp32 results
        _att("blocks_ragged", "blocks", 5, 3001, True, True, 8, 8, 128, "f32", "rows", 9, 128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges: 1 to 49152 tokens, widths to 4096, every type, norm, gate and layout; heads of 16 to
    128, sequences of 1 to 16384 tokens, 1 to 64 chosen blocks."""
    op = rng.choice(["norm", "norm", "attention", "attention", "select", "blocks", "blocks"])
    if op == "norm":
        m, n = _log_int(rng, 1, 49152), rng.choice([768, 1024, 4096, _log_int(rng, 16, 4096)])
        m = min(m, 49152 * 1024 // n)
        c = _norm("", m, n, rng.choice(["f32", "i8"]), rng.choice(["f32", "f32", "i8", "none"]),
                  rng.choice(["none", "layer", "rms"]), rng.choice(["none", "channel", "token", "element"]),
                  rng.choice(["layer", "rms"]), rng.choice([1.0, 0.5, 1.7]), rng.choice(["", "h", "u", "hu"]),
                  rng.choice(["rows", "tiles"]))
    else:
        hd = rng.choice([64, 64, 64, 32, 128, 16, 48, 80, 96])
        nkv = rng.choice([1, 2, 4, 8, 12])
        nh = nkv * rng.choice([1, 1, 2, 4] if nkv <= 4 else [1])
        s = _log_int(rng, 1, 8192) if op == "attention" else _log_int(rng, 64, 16384)
        cost = lambda s: nh * max(hd, 64) / 64 * s * (s if op == "attention" else min(s, 2048))  # noqa: E731
        while cost(s) > 4e8:
            s = s * 2 // 3
        b = max(1, min(128, int(4e8 / cost(s)), 49152 // s))
        b = _log_int(rng, 1, b)
        ragged = b > 1 and rng.random() < 0.6
        c = _att("", op, b, s, ragged, rng.random() < 0.3, nh, nkv, hd, rng.choice(["i8", "i8", "f32"]),
                 rng.choice(["rows", "tiles"]))
        if op != "attention":
            c.update(top_k=_log_int(rng, 1, 32), qb=rng.choice([16, 32, 64, 64, 128]))
    del c["name"]
    return c


# --- inputs -----------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 29)


def _bf(v):
    """v rounded up to 8 significant bits, a bfloat16, so that a code times it is rounded once."""
    m, e = math.frexp(v)
    return math.ldexp(math.ceil(m * 256) / 256, e)


def _tiles(x):
    """An int8 [m, k] tensor in the tile layout, zeros for padding."""
    m, k = x.shape
    rb, cb = (m + 15) // 16, (k + 31) // 32
    p = torch.zeros((rb * 16, cb * 32), dtype=x.dtype, device=x.device)
    p[:m, :k] = x
    return p.reshape(rb, 16, cb, 32).permute(0, 2, 1, 3).contiguous()


def _rows(x, m, k):
    """The [m, k] tensor that a tile-layout tensor holds."""
    rb, cb = x.shape[:2]
    return x.permute(0, 2, 1, 3).reshape(rb * 16, cb * 32)[:m, :k]


def _laid(case, x):
    return _tiles(x) if case["layout"] == "tiles" else x


def _y_tiles(case, m, n):
    """int8 results come in the case's layout where that leaves no padding."""
    return case["layout"] == "tiles" and m % 16 == 0 and n % 32 == 0


def _lengths(case, seed):
    """Lengths of the sequences and their valid keys."""
    b, s = case["b"], case["s"]
    g = torch.Generator().manual_seed(int(seed) * 911 + 5)
    if case["ragged"]:  # the same lengths for every seed, in another order
        lens = torch.randint(1, s + 1, (b,), generator=torch.Generator().manual_seed(1000 * b + s))
        lens[0] = s
        if b > 1:
            lens[1] = 1
        lens = lens[torch.randperm(b, generator=g)].tolist()
    else:
        lens = [s] * b
    keys = list(lens)
    if case["masked"]:
        keys = [int(torch.randint(1, n + 1, (1,), generator=g)) for n in lens]
        if b > 2:
            keys[2] = 0
    return lens, keys


def _activations(m, cols, g):
    """int8 codes [m, cols]: a part of each token's own and one that changes every 96 tokens or so."""
    x = torch.randn((m, cols), generator=g, device="cuda")
    topic = torch.randn((m // 96 + 1, cols), generator=g, device="cuda")
    x.mul_(0.85).add_(topic.mul_(0.53)[torch.arange(m, device="cuda") // 96])
    return x.mul_(127 / 4).round_().clamp_(-127, 127).to(torch.int8)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    if case["op"] == "norm":
        m, n = case["m"], case["n"]
        f = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
        codes = lambda: f(m, n).mul_(127 / 4).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
        s["y_scale"], s["r_scale"], s["out_scale"] = 0.02, 0.03, _bf(4.2 / 127)
        s["y"] = _laid(case, codes()) if case["y"] == "i8" else f(m, n).mul_(0.7)
        s["r"] = None if case["r"] == "none" else _laid(case, codes()) if case["r"] == "i8" else f(m, n)
        shape = {"none": None, "channel": (n,), "token": (m, 1), "element": (m, n)}[case["gate"]]
        s["gate"] = None if shape is None else torch.sigmoid(f(*shape))
        s["gamma"], s["beta"] = f(n).mul_(0.1).add_(1), f(n).mul_(0.05)
        s["pgamma"], s["pbeta"] = f(n).mul_(0.1).add_(1), f(n).mul_(0.05)
        s["value"] = torch.tensor(s["out_scale"], dtype=torch.bfloat16)
        return s
    lens, keys = _lengths(case, seed)
    m, nh, nkv, hd = sum(lens), case["nh"], case["nkv"], case["hd"]
    cols = (nh + 2 * nkv) * hd
    x = _activations(m, cols, g)
    start = [0]
    for n in lens:
        start.append(start[-1] + n)
    b, longest = len(lens), max(lens)
    s.update(m=m, cols=cols, longest=longest, x=_laid(case, x), x_scale=0.04)
    s["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
    s["keys"] = torch.tensor(keys, dtype=torch.int32, device="cuda") if case["masked"] else None
    # where the plain form finds token i of sequence b (past a sequence's end: any token), and which places are real
    at = torch.arange(longest, device="cuda")[None, :]
    first, count = s["start"][:-1, None].long(), torch.tensor(lens, device="cuda")[:, None]
    s["at"] = (first + at).clamp_(max=m - 1)
    s["real"] = at < count
    s["nkeys"] = torch.tensor(keys, device="cuda")
    # an average of about n keys: of a value's own spread, the largest of which is about 4 deviations
    seen = [min(n, case["top_k"] * BLOCK) if case["op"] == "blocks" else n for n in keys]
    typical = sorted(max(n, 1) for n in seen)[0]
    s["out_scale"] = _bf(s["x_scale"] * (18 + 109 / typical ** 0.5) / 127)
    s["value"] = torch.tensor(s["out_scale"], dtype=torch.bfloat16)
    return s


# --- one pass ---------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _own_norm(state) if case["op"] == "norm" else _own_attention(state)
    return _plain_norm(state) if case["op"] == "norm" else _plain_attention(state)


def _own_norm(s):
    import paper_2211_07715_amd as sl
    c = s["case"]
    layout = sl.LAYOUT_T16X32 if c["layout"] == "tiles" else sl.LAYOUT_ROWS
    kinds = {"none": sl.NORM_NONE, "layer": sl.NORM_LAYER, "rms": sl.NORM_RMS}
    h, u, q = sl.residual_norm(
        s["y"], s["gamma"], s["beta"] if c["norm"] == "layer" else None, norm=kinds[c["norm"]], eps=EPS,
        y_scale=s["y_scale"], residual=s["r"], residual_scale=c["rscale"], r_scale=s["r_scale"], gate=s["gate"],
        post_norm=kinds[c["post"]], post_gamma=s["pgamma"] if c["post"] != "none" else None,
        post_beta=s["pbeta"] if c["post"] == "layer" else None, keep_sum="h" in c["keep"], keep_norm="u" in c["keep"],
        out_scale=s["out_scale"], y_layout=layout if c["y"] == "i8" else sl.LAYOUT_ROWS,
        r_layout=layout if c["r"] == "i8" else sl.LAYOUT_ROWS,
        q_layout=layout if _y_tiles(c, c["m"], c["n"]) else sl.LAYOUT_ROWS, shape=(c["m"], c["n"]))
    out = {"q": q * s["value"]}
    if h is not None:
        out["h"] = h
    if u is not None:
        out["u"] = u
    return out


def _own_attention(s):
    import paper_2211_07715_amd as sl
    c = s["case"]
    layout = sl.LAYOUT_T16X32 if c["layout"] == "tiles" else sl.LAYOUT_ROWS
    blocks, out = None, {}
    if c["op"] != "attention":
        blocks = sl.select_blocks(s["x"], s["start"], s["longest"], c["nh"], c["hd"], c["top_k"], n_kv_heads=c["nkv"],
                                  query_block=c["qb"], key_len=s["keys"], x_layout=layout, m_tokens=s["m"])
        out["blocks"] = blocks
        if c["op"] == "select":
            return out
    whole = _y_tiles(c, s["m"], c["nh"] * c["hd"])
    kind = sl.EPI_I8 if c["kind"] == "i8" else sl.EPI_F32
    y = sl.attention(s["x"], s["x_scale"], s["start"], s["longest"], c["nh"], c["hd"], n_kv_heads=c["nkv"],
                     key_len=s["keys"], kind=kind, out_scale=s["out_scale"], blocks=blocks, query_block=c["qb"] or 64,
                     x_layout=layout, y_layout=layout if whole and kind == sl.EPI_I8 else sl.LAYOUT_ROWS,
                     m_tokens=s["m"])
    out["y"] = y * s["value"] if c["kind"] == "i8" else y
    return out


def _codes(x, scale):
    return torch.clamp(torch.round(x * (1.0 / scale)), -127, 127)


def _plain_one(x, kind, gamma, beta):
    if kind == "layer":
        d = x - x.mean(1, keepdim=True)
        return d / torch.sqrt((d * d).mean(1, keepdim=True) + EPS) * gamma + beta
    return x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * gamma


def _plain_norm(s):
    c = s["case"]
    m, n = c["m"], c["n"]

    def real(x, is_codes, scale):
        if not is_codes:
            return x
        return (_rows(x, m, n) if c["layout"] == "tiles" else x).float() * scale

    t = real(s["y"], c["y"] == "i8", s["y_scale"])
    if c["post"] != "none":
        t = _plain_one(t, c["post"], s["pgamma"], s["pbeta"])
    if s["gate"] is not None:
        t = t * s["gate"]
    h = t if s["r"] is None else real(s["r"], c["r"] == "i8", s["r_scale"]) * c["rscale"] + t
    u = _plain_one(h, c["norm"], s["gamma"], s["beta"])
    q = _codes(u, s["out_scale"]).to(torch.bfloat16) * s["value"]
    out = {"q": _tiles(q) if _y_tiles(c, m, n) else q}
    if "h" in c["keep"]:
        out["h"] = h
    if "u" in c["keep"]:
        out["u"] = u
    return out


def _plain_attention(s):
    c = s["case"]
    b, n, nh, nkv, hd = c["b"], s["longest"], c["nh"], c["nkv"], c["hd"]
    x = (_rows(s["x"], s["m"], s["cols"]) if c["layout"] == "tiles" else s["x"])[s["at"]].float()  # [b, n, cols]
    x = x.reshape(b, n, nh + 2 * nkv, hd).transpose(1, 2)
    q, k, v = x[:, :nh], x[:, nh:nh + nkv], x[:, nh + nkv:]
    if nkv != nh:
        k, v = k.repeat_interleave(nh // nkv, dim=1), v.repeat_interleave(nh // nkv, dim=1)
    key_ok = torch.arange(n, device=x.device)[None, :] < s["nkeys"][:, None]  # [b, n]
    out, scale = {}, s["x_scale"] ** 2 / math.sqrt(hd)
    if c["op"] == "attention":
        p = (q @ k.transpose(2, 3).contiguous()).mul_(scale)
        p = _softmax(p, key_ok[:, None, None, :])
        o = p @ v
    else:
        qb, top = c["qb"], c["top_k"]
        blocks = _plain_select(s, q, k, key_ok)
        out["blocks"] = blocks
        if c["op"] == "select":
            return out
        nq, nb = blocks.shape[2], -(-n // BLOCK)
        pad = lambda t, to: torch.nn.functional.pad(t, (0, 0, 0, to - n))  # noqa: E731
        idx = blocks.long().clamp(min=0)  # [b, nh, nq, top]
        pick = idx[..., None] * BLOCK + torch.arange(BLOCK, device=x.device)  # positions of the chosen keys
        ok = (pick < s["nkeys"][:, None, None, None, None]) & (blocks >= 0)[..., None]
        ok = ok.reshape(b, nh, nq, 1, top * BLOCK)
        take = idx.reshape(b, nh, nq * top, 1, 1).expand(-1, -1, -1, BLOCK, hd)

        def chosen(t):
            t = pad(t, nb * BLOCK).reshape(b, nh, nb, BLOCK, hd)
            return torch.gather(t, 2, take).reshape(b, nh, nq, top * BLOCK, hd)

        p = (pad(q, nq * qb).reshape(b, nh, nq, qb, hd) @ chosen(k).transpose(3, 4).contiguous()).mul_(scale)
        o = (_softmax(p, ok) @ chosen(v)).reshape(b, nh, nq * qb, hd)[:, :, :n]
    o = (o * s["x_scale"]).transpose(1, 2).reshape(b, n, nh * hd)[s["real"]]  # [m, nh hd]
    if c["kind"] == "i8":
        o = _codes(o, s["out_scale"]).to(torch.bfloat16) * s["value"]
        o = _tiles(o) if _y_tiles(c, s["m"], nh * hd) else o
    out["y"] = o
    return out


def _softmax(p, ok):
    """Softmax of the last dimension over the places that are ok; zeros where none is. (p is overwritten)"""
    p = p.masked_fill_(~ok, -math.inf)
    top = p.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = p.sub_(top).exp_()
    return p.div_(p.sum(-1, keepdim=True).clamp_(min=1e-30))


def _plain_select(s, q, k, key_ok):
    """The chosen blocks. Scores are whole numbers of up to 35 bits: in 64-bit floats their sums are exact."""
    c = s["case"]
    b, n, nh, hd, qb, top = c["b"], s["longest"], c["nh"], c["hd"], c["qb"], c["top_k"]
    nq, nb = -(-n // qb), -(-n // BLOCK)
    pad = torch.nn.functional.pad
    ks = pad(k * key_ok[:, None, :, None], (0, 0, 0, nb * BLOCK - n)).reshape(b, nh, nb, BLOCK, hd).sum(3)
    qs = pad(q * s["real"][:, None, :, None], (0, 0, 0, nq * qb - n)).reshape(b, nh, nq, qb, hd).sum(3)
    first = torch.arange(nb, device=q.device) * BLOCK
    have = (s["nkeys"][:, None] - first[None, :]).clamp(0, BLOCK)  # keys of each block [b, nb]
    ks = torch.round(ks * BLOCK / have.clamp(min=1)[:, None, :, None])
    score = qs.double() @ ks.double().transpose(2, 3).contiguous()  # [b, nh, nq, nb]
    score = score.masked_fill(have[:, None, None, :] == 0, -math.inf)
    best = torch.sort(score, dim=3, descending=True, stable=True).indices[..., :top]
    if nb < top:
        best = pad(best, (0, top - nb), value=nb)
    count = (have > 0).sum(1)  # blocks of each sequence
    rows = (torch.arange(nq, device=q.device) * qb)[None, :] < s["real"].sum(1)[:, None]
    gone = (torch.arange(top, device=q.device)[None, None, None, :] >= count[:, None, None, None]) | ~rows[:, None, :, None]
    best = best.masked_fill(gone, nb).sort(dim=3).values
    return best.masked_fill(best == nb, -1).to(torch.int32)


# --- what a pass cannot do without, and what it has to give -----------------

def work(case):
    if case["op"] == "norm":
        m, n = case["m"], case["n"]
        e = {"f32": 4, "i8": 1, "none": 0}
        each = e[case["y"]] + e[case["r"]] + 1 + 4 * len(case["keep"]) + (4 if case["gate"] == "element" else 0)
        more = 4 * n * (2 + (2 if case["post"] != "none" else 0) + (1 if case["gate"] == "channel" else 0))
        return {"bytes": float(m * n * each + more + (4 * m if case["gate"] == "token" else 0)), "flops": 20.0 * m * n}
    # (ragged sequences count as half their longest, their valid keys as half of them)
    b, nh, nkv, hd = case["b"], case["nh"], case["nkv"], case["hd"]
    s = case["s"] / 2 if case["ragged"] else case["s"]
    keys = s / 2 if case["masked"] else s
    m = b * s
    lists = 4.0 * b * nh * -(-case["s"] // case["qb"]) * case["top_k"] if case["op"] != "attention" else 0.0
    pairs = m * nh * (min(keys, case["top_k"] * BLOCK) if case["op"] == "blocks" else keys)
    if case["op"] == "select":
        return {"bytes": m * (nh + nkv) * hd + lists, "flops": 2.0 * m / case["qb"] * nh * keys / BLOCK * hd}
    y = m * nh * hd * (1 if case["kind"] == "i8" else 4)
    return {"bytes": m * (nh + 2 * nkv) * hd + y + lists, "flops": 4.0 * pairs * hd}


def exact(case, seed):
    """The results in 64 bits, from the definitions, a sequence and a head at a time."""
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, s)
    lens, keys = _lengths(case, seed)
    nh, nkv, hd, m = case["nh"], case["nkv"], case["hd"], s["m"]
    if sum(n * n for n in lens) * nh * hd > 3e12:
        return None
    x = (_rows(s["x"], m, s["cols"]) if case["layout"] == "tiles" else s["x"]).reshape(m, nh + 2 * nkv, hd)
    o = torch.zeros((m, nh, hd), dtype=torch.float64, device=x.device)
    lists, top, qb = None, case["top_k"], case["qb"]
    if case["op"] != "attention":
        lists = torch.full((len(lens), nh, -(-s["longest"] // qb), top), -1, dtype=torch.int32, device=x.device)
    first = 0
    for i, (n, nk) in enumerate(zip(lens, keys)):
        part, first = x[first:first + n], first + n
        for h in range(nh):
            kv = nh + h // (nh // nkv)
            qi, ki = part[:, h], part[:nk, kv]
            use = None
            if lists is not None and nk:
                use = _exact_lists(qi.long(), ki.long(), qb, top)  # [query blocks, blocks] chosen or not
                count = min(top, use.shape[1])
                lists[i, h, :use.shape[0], :count] = use.nonzero()[:, 1].reshape(use.shape[0], count).to(torch.int32)
            if case["op"] == "select" or nk == 0:
                continue
            z = (qi.double() @ ki.double().t()) * (s["x_scale"] ** 2 / math.sqrt(hd))
            if use is not None:
                seen = use[torch.arange(n, device=x.device) // qb][:, torch.arange(nk, device=x.device) // BLOCK]
                z = torch.where(seen, z, torch.full_like(z, -math.inf))
            o[first - n:first, h] = torch.softmax(z, dim=1) @ (part[:nk, kv + nkv].double() * s["x_scale"])
    out = {} if lists is None else {"blocks": lists}
    if case["op"] != "select":
        o = o.reshape(m, nh * hd)
        if case["kind"] == "i8":
            o = torch.round(o / s["out_scale"]).clamp(-127, 127) * s["out_scale"]
            o = _tiles(o) if _y_tiles(case, m, nh * hd) else o
        out["y"] = o
    return out


def _exact_lists(q, k, qb, top):
    """Chosen blocks by whole-number scores: the pooled sums are multiplied out in 64-bit integers."""
    qs = torch.stack([t.sum(0) for t in q.split(qb)])
    ks = []
    for t in k.split(BLOCK):
        total, n = t.sum(0) * BLOCK, t.shape[0]
        low, twice = torch.div(total, n, rounding_mode="floor"), 2 * (total % n)
        ks.append(low + ((twice > n) | ((twice == n) & (low % 2 == 1))).long())  # half to even
    ks = torch.stack(ks)
    use = torch.zeros((qs.shape[0], ks.shape[0]), dtype=torch.bool, device=q.device)
    for i, part in enumerate(qs.split(64)):
        score = (part[:, None, :] * ks[None]).sum(2)
        order = torch.argsort(-score, dim=1, stable=True)[:, :top]
        use[64 * i:64 * i + part.shape[0]].scatter_(1, order, True)
    return use


def _exact_norm(c, s):
    m, n = c["m"], c["n"]

    def real(x, is_codes, scale):
        if is_codes and c["layout"] == "tiles":
            x = _rows(x, m, n)
        return x.double() * (scale if is_codes else 1.0)

    def normed(x, kind, gamma, beta):
        mean = x.mean(1, keepdim=True) if kind == "layer" else 0.0
        var = (x - mean).square().mean(1, keepdim=True)
        x = (x - mean) * (var + EPS).rsqrt() * gamma.double()
        return x + beta.double() if kind == "layer" else x

    h = real(s["y"], c["y"] == "i8", s["y_scale"])
    if c["post"] != "none":
        h = normed(h, c["post"], s["pgamma"], s["pbeta"])
    if s["gate"] is not None:
        h = h * s["gate"].double()
    if s["r"] is not None:
        h = h + c["rscale"] * real(s["r"], c["r"] == "i8", s["r_scale"])
    u = normed(h, c["norm"], s["gamma"], s["beta"])
    q = torch.round(u / s["out_scale"]).clamp(-127, 127) * s["out_scale"]
    out = {"q": _tiles(q) if _y_tiles(c, m, n) else q}
    if "h" in c["keep"]:
        out["h"] = h
    if "u" in c["keep"]:
        out["u"] = u
    return out
