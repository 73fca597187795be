"""What the speed of the operators of a decoder's key-value cache is measured on:
``cache_append`` and ``cache_attention``, as a serving program of an int8 decoder
calls them.

``own`` false: every operator in its plain form, elementary torch operations in
32 bits (angles of positions in 64). ``own`` true: the calls of this package. A
case is a dict of plain values; ``op`` says what one pass is:

    append     one ``cache_append``: the output of a fused QKV linear, its queries
               and keys rotated by position, goes to the query codes that
               attention reads and to the pages of an int8 cache
    attend     one ``cache_attention``: the newest ``new`` tokens of each sequence
               over the keys and values that its pages hold, each up to its own
               place (``causal``) or over all of them (an encoder's states)

``b`` sequences hold ``s`` tokens each, of which the last ``new`` are the pass's
(``ragged``: numbers of both drawn from 1 on, one sequence idle: nothing cached);
without ``causal`` the two are apart. Pages of ``ps`` tokens lie in any order. A
page holds, for each key-value head, its keys [ps][hd] and then, for each, its
values [ps / 16][hd][16]: 16 tokens' values of a feature lie together. ``layout``
is that of the int8 activations: ``rows`` or ``tiles`` (16 tokens x 32 features).
Int8 results, the cache among them, are returned as the values they stand for, in
bfloat16.
"""
import math

import torch

own = False

ROWS, TILES = 0, 1  # the package's numbers of the two layouts
F32, I8 = 1, 3      # and of its fp32 and int8 results
HALF, INTERLEAVED = 1, 2  # and of the order of a rotated pair's features


def _app(name, b, new, s, ragged, nh, nkv, hd, ps, x, layout, rope, rot, far=0):
    return dict(name=name, op="append", b=b, new=new, s=s, ragged=ragged, causal=True, nh=nh, nkv=nkv, hd=hd, ps=ps, x=x,
                layout=layout, rope=rope, rot=rot, far=far)


def _att(name, b, new, s, ragged, causal, nh, nkv, hd, ps, kind, layout):
    return dict(name=name, op="attend", b=b, new=new, s=s, ragged=ragged, causal=causal, nh=nh, nkv=nkv, hd=hd, ps=ps,
                kind=kind, layout=layout)


def listed():
    return [
        # the smallest: one token of one sequence
        _app("append_b1", 1, 1, 100, False, 12, 12, 64, 16, "i8", "rows", "half", 64),
        # a step of 64 sequences early in their answers, from a linear's fp32 output
        _app("append_b64", 64, 1, 100, True, 32, 8, 128, 16, "f32", "rows", "half", 128),
        # unpadded prompts of 1 to 384 tokens behind cached ones, part of each head rotated, far positions
        _app("append_ragged", 24, 384, 500, True, 12, 12, 64, 16, "i8", "tiles", "interleaved", 32, 100000),
        # long prompts, whole
        _app("append_b4_s4096", 4, 4096, 4096, False, 32, 8, 128, 64, "f32", "rows", "half", 128),
        # batch-1 latency of a step
        _att("step_b1_s128", 1, 1, 128, False, True, 12, 12, 64, 16, "i8", "rows"),
        # throughput serving, key and value heads shared by 4 query heads
        _att("step_b64_s4096", 64, 1, 4096, False, True, 32, 8, 128, 64, "i8", "rows"),
        # sequences of 1 to 3001 tokens, one idle, fp32 results
        _att("step_ragged", 24, 1, 3001, True, True, 8, 8, 96, 16, "f32", "rows"),
        # one very long document
        _att("step_b1_s131072", 1, 1, 131072, False, True, 32, 8, 128, 256, "i8", "rows"),
        # a step's attention to an encoder's states
        _att("cross_step_b32_s384", 32, 1, 384, False, False, 12, 12, 64, 64, "i8", "tiles"),
        # 128 tokens at once over an encoder's states
        _att("cross_b32_s384", 32, 128, 384, False, False, 12, 12, 64, 64, "i8", "tiles"),
        # prompts in pieces: 1 to 512 new tokens behind up to 2048
        _att("prompt_ragged", 16, 512, 2048, True, True, 12, 12, 64, 32, "f32", "rows"),
        # a long prompt, whole
        _att("prompt_s8192", 1, 8192, 8192, False, True, 16, 4, 64, 64, "i8", "rows"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """A case of the same ranges: heads of 16 to 128 features, 1 to 8 query heads a key-value head, pages of 16 to 256
    tokens; 1 to 131072 cached tokens and 1 to 8192 new ones a sequence, up to 128 sequences, every type and layout."""
    op = rng.choice(["append", "append", "attend", "attend", "attend"])
    hd = rng.choice([64, 64, 128, 128, 32, 16, 48, 80, 96])
    nkv = rng.choice([1, 2, 4, 8, 12])
    nh = nkv * rng.choice([1, 2, 4, 8] if nkv <= 4 else [1, 2, 4])
    ps = rng.choice([16, 32, 64, 64, 128, 256])
    layout = rng.choice(["rows", "rows", "tiles"])
    if op == "append":
        x = rng.choice(["f32", "i8"])
        rope = rng.choice(["none", "half", "half", "interleaved"])
        new = rng.choice([1, 1, _log_int(rng, 2, 4096)])
        most = max(1, int(16384 * 6144 / (new * (nh + 2 * nkv) * hd)))
        b = _log_int(rng, 1, min(64, most))
        s = new + _log_int(rng, 1, 300)
        rot = 0 if rope == "none" else rng.choice([hd, hd, hd // 2, 2 * rng.randint(1, hd // 2)])
        c = _app("", b, new, s, b > 1 and rng.random() < 0.5, nh, nkv, hd, ps, x, layout if x == "i8" else "rows", rope,
                 rot, rng.choice([0, 0, 100000]))
    else:
        causal = rng.random() < 0.7
        new = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 4096)])
        s = _log_int(rng, max(new, 16) if causal else 16, 131072 if new < 9 else 8192)
        while new * s * nh * max(hd, 64) > 8192 * 8192 * 16 * 64 / 2 or s * nkv * hd > 131072 * 8 * 128:
            s = max(s * 2 // 3, new if causal else 1)
            if causal and s == new:
                new = max(1, new * 2 // 3)
        most = min(64 * 4096 * 8 * 128 / (s * nkv * hd), 8192 * 8192 * 16 * 64 / 2 / (new * s * nh * max(hd, 64)))
        b = _log_int(rng, 1, max(1, min(128, int(most))))
        c = _att("", b, new, s, b > 1 and rng.random() < 0.5, causal, nh, nkv, hd, ps, rng.choice(["i8", "i8", "f32"]),
                 layout)
    del c["name"]
    return c


# --- inputs -----------------------------------------------------------------

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


def _whole(case, m):
    """int8 results come in the case's layout where that leaves no padding."""
    return case["layout"] == "tiles" and m % 16 == 0 and case["nh"] * case["hd"] % 32 == 0


def _lengths(case, seed):
    """New and cached tokens of every sequence (the cached ones include the new ones where that is causal)."""
    b, new, s = case["b"], case["new"], case["s"]
    if not case["ragged"]:
        return [new] * b, [s] * b
    g = torch.Generator().manual_seed(1000 * b + s)  # the same numbers for every seed, in another order
    news = torch.randint(1, new + 1, (b,), generator=g).tolist()
    lens = torch.randint(1, s + 1, (b,), generator=g).tolist()
    news[0], lens[0] = new, s
    news[1], lens[1] = 1, 1
    if case["causal"]:
        lens = [max(n, t) for n, t in zip(news, lens)]
    if b > 2:
        news[2], lens[2] = 1, 0
    order = torch.randperm(b, generator=torch.Generator().manual_seed(int(seed) * 911 + 5)).tolist()
    return [news[i] for i in order], [lens[i] for i in order]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 31)
    news, lens = _lengths(case, seed)
    b, nh, nkv, hd, ps = case["b"], case["nh"], case["nkv"], case["hd"], case["ps"]
    m, dev = sum(news), "cuda"
    f = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    codes = lambda *shape: f(*shape).mul_(127 / 4).round_().clamp_(-127, 127).to(torch.int8)  # noqa: E731
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    # pages in any order; entries behind a sequence's last page name none
    count = [-(-n // ps) for n in lens]
    per, pages = max(max(count), 1), max(sum(count), 1)
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    table = torch.full((b, per), -1, dtype=torch.int32, device=dev)
    have = torch.arange(per, device=dev)[None, :] < i32(count)[:, None]
    table[have] = order[:sum(count)]
    start = [0]
    for n in news:
        start.append(start[-1] + n)
    # (scales of 8 bits: a code times one is rounded once; and no code of v's scale is halfway between two of q's or k's)
    s = {"case": case, "m": m, "longest": max(max(lens), 1), "most_new": max(news), "table": table, "start": i32(start),
         "len": i32(lens), "cache": codes(pages, 2, nkv, ps, hd), "q_scale": 165 / 4096, "k_scale": 205 / 4096,
         "v_scale": 123 / 4096}
    # which sequence a new token is of, and its place there (as the plain form looks them up)
    s["seq"] = torch.repeat_interleave(torch.arange(b, device=dev), i32(news).long())
    nth = torch.arange(m, device=dev) - s["start"].long()[s["seq"]]
    s["nth"], s["news"] = nth, i32(news).long()
    s["slot"] = s["len"].long()[s["seq"]] - s["news"][s["seq"]] + nth
    if case["op"] == "append":
        cols = (nh + 2 * nkv) * hd
        if case["x"] == "i8":
            x = codes(m, cols)
            s["x"], s["x_scale"] = _tiles(x) if case["layout"] == "tiles" else x, s["v_scale"]
        else:
            s["x"], s["x_scale"] = f(m, cols).mul_(127 * s["v_scale"] / 4), 1.0
        rot = case["rot"]
        # scaled for long contexts where positions are far: slower angles, and a factor on both
        slow, s["factor"] = (4.0, 1.1386) if case["far"] else (1.0, 1.0)
        at = torch.arange(0, rot, 2, dtype=torch.float64, device=dev)
        s["freq"] = (10000.0 ** (-at / max(rot, 1)) / slow).float() if rot else None
        s["pos"] = (s["slot"] + case["far"]).to(torch.int32) if case["far"] else None
        s["kv_value"] = torch.tensor([s["k_scale"], s["v_scale"]], dtype=torch.bfloat16, device=dev).reshape(2, 1, 1, 1)
        s["q_value"] = torch.tensor(s["q_scale"], dtype=torch.bfloat16)
    else:
        q = codes(m, nh * hd)
        s["q"] = _tiles(q) if case["layout"] == "tiles" else q
        typical = sorted(max(n, 1) for n in lens)[0]
        s["out_scale"] = _bf(s["v_scale"] * (18 + 109 / typical ** 0.5) / 127)
        s["value"] = torch.tensor(s["out_scale"], dtype=torch.bfloat16)
    return s


# --- one pass ---------------------------------------------------------------

def run(state):
    if own:
        return _own_append(state) if state["case"]["op"] == "append" else _own_attend(state)
    return _plain_append(state) if state["case"]["op"] == "append" else _plain_attend(state)


def _own_append(s):
    import paper_2211_07715_amd as sl
    c = s["case"]
    layout = sl.LAYOUT_T16X32 if c["layout"] == "tiles" else sl.LAYOUT_ROWS
    rope = {"none": sl.ROPE_NONE, "half": sl.ROPE_HALF, "interleaved": sl.ROPE_INTERLEAVED}[c["rope"]]
    q = sl.cache_append(s["x"], s["cache"], s["table"], s["start"], s["len"], s["most_new"], c["nh"],
                        x_scale=s["x_scale"], q_scale=s["q_scale"], k_scale=s["k_scale"], v_scale=s["v_scale"], rope=rope,
                        inv_freq=s["freq"], rope_factor=s["factor"], positions=s["pos"],
                        x_layout=layout if c["x"] == "i8" else sl.LAYOUT_ROWS,
                        q_layout=layout if _whole(c, s["m"]) else sl.LAYOUT_ROWS, m_tokens=s["m"])
    return {"q": q * s["q_value"], "cache": s["cache"] * s["kv_value"]}


def _own_attend(s):
    import paper_2211_07715_amd as sl
    c = s["case"]
    layout = sl.LAYOUT_T16X32 if c["layout"] == "tiles" else sl.LAYOUT_ROWS
    kind = sl.EPI_I8 if c["kind"] == "i8" else sl.EPI_F32
    y = sl.cache_attention(s["q"], s["cache"], s["table"], s["start"], s["len"], s["most_new"], s["longest"], c["nh"],
                           q_scale=s["q_scale"], k_scale=s["k_scale"], v_scale=s["v_scale"], causal=c["causal"], kind=kind,
                           out_scale=s["out_scale"], q_layout=layout,
                           y_layout=layout if kind == sl.EPI_I8 and _whole(c, s["m"]) else sl.LAYOUT_ROWS,
                           m_tokens=s["m"])
    return {"y": y * s["value"] if c["kind"] == "i8" else y}


def _codes(x, scale):
    return torch.clamp(torch.round(x * (1.0 / scale)), -127, 127)


def _plain_append(s):
    c = s["case"]
    m, nh, nkv, hd, ps, rot = s["m"], c["nh"], c["nkv"], c["hd"], c["ps"], c["rot"]
    x = s["x"]
    if c["x"] == "i8":
        x = (_rows(x, m, (nh + 2 * nkv) * hd) if c["layout"] == "tiles" else x).float() * s["x_scale"]
    x = x.reshape(m, nh + 2 * nkv, hd)
    qk, v = x[:, :nh + nkv], x[:, nh + nkv:]
    if rot:
        pos = s["slot"] if s["pos"] is None else s["pos"]
        angle = pos.double()[:, None] * s["freq"].double()[None, :]
        cos, sin = (angle.cos() * s["factor"]).float()[:, None], (angle.sin() * s["factor"]).float()[:, None]
        if c["rope"] == "half":
            a, d = qk[..., :rot // 2], qk[..., rot // 2:rot]
            turned = torch.cat([a * cos - d * sin, d * cos + a * sin], 2)
        else:
            a, d = qk[..., 0:rot:2], qk[..., 1:rot:2]
            turned = torch.stack([a * cos - d * sin, d * cos + a * sin], 3).reshape(m, nh + nkv, rot)
        qk = torch.cat([turned, qk[..., rot:]], 2)
    k, v = _codes(qk[:, nh:], s["k_scale"]).to(torch.int8), _codes(v, s["v_scale"]).to(torch.int8)
    put = s["slot"] >= 0
    at, seq = s["slot"].clamp(min=0), s["seq"]
    page = s["table"][seq, at // ps].long()
    page, at, k, v = page[put], at[put] % ps, k[put], v[put]
    s["cache"][:, 0].index_put_((page[:, None], torch.arange(nkv, device=x.device)[None, :], at[:, None]), k)
    values = s["cache"][:, 1].view(-1, nkv, ps // 16, hd, 16)
    values[page, :, at // 16, :, at % 16] = v
    q = _codes(qk[:, :nh], s["q_scale"]).reshape(m, nh * hd).to(torch.bfloat16) * s["q_value"]
    return {"q": _tiles(q) if _whole(c, m) else q, "cache": s["cache"] * s["kv_value"]}


def _plain_attend(s):
    c = s["case"]
    b, nh, nkv, hd, ps, n, m = c["b"], c["nh"], c["nkv"], c["hd"], c["ps"], s["most_new"], s["m"]
    g, per = nh // nkv, s["table"].shape[1]
    q = _rows(s["q"], m, nh * hd) if c["layout"] == "tiles" else s["q"]
    at = torch.arange(n, device=q.device)[None, :]
    q = q[(s["start"].long()[:-1, None] + at).clamp_(max=m - 1)].float()  # [b, n, nh hd]
    q = q.reshape(b, n, nkv, g, hd).permute(0, 2, 3, 1, 4).reshape(b, nkv, g * n, hd)
    pages = s["cache"][s["table"].long().clamp(min=0)]  # [b, per, 2, nkv, ps, hd]
    k = pages[:, :, 0].permute(0, 2, 4, 1, 3).reshape(b, nkv, hd, per * ps).float()
    v = pages[:, :, 1].reshape(b, per, nkv, ps // 16, hd, 16).permute(0, 2, 1, 3, 5, 4)
    v = v.reshape(b, nkv, per * ps, hd).float()
    p = (q @ k).mul_(s["q_scale"] * s["k_scale"] / math.sqrt(hd)).reshape(b, nkv, g, n, per * ps)
    last = s["len"].long()[:, None].expand(b, n)  # keys that a query sees
    if c["causal"]:
        last = last - s["news"][:, None] + at + 1
    seen = torch.arange(per * ps, device=q.device)[None, None, :] < torch.minimum(last, s["len"].long()[:, None])[..., None]
    p = p.masked_fill_(~seen[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True).clamp_(min=-3e38)).exp_()
    p = p.div_(p.sum(-1, keepdim=True).clamp_(min=1e-30))
    o = (p.reshape(b, nkv, g * n, per * ps) @ v).mul_(s["v_scale"])
    o = o.reshape(b, nkv, g, n, hd).permute(0, 3, 1, 2, 4).reshape(b, n, nh * hd)
    o = o[s["seq"], s["nth"]]  # [m, nh hd]
    if c["kind"] == "i8":
        o = _codes(o, s["out_scale"]).to(torch.bfloat16) * s["value"]
        o = _tiles(o) if _whole(c, m) else o
    return {"y": o}


# --- what a pass cannot do without, and what it has to give -----------------

def work(case):
    news, lens = _lengths(case, 0)
    m, nh, nkv, hd = sum(news), case["nh"], case["nkv"], case["hd"]
    if case["op"] == "append":
        cols = (nh + 2 * nkv) * hd
        return {"bytes": float(m * cols * ((4 if case["x"] == "f32" else 1) + 1)), "flops": float(m * cols * 6)}
    pairs = 0
    for n, t in zip(news, lens):
        pairs += sum(max(0, t - n + i + 1) for i in range(n)) if case["causal"] else n * t
    y = m * nh * hd * (1 if case["kind"] == "i8" else 4)
    return {"bytes": float(sum(lens) * nkv * hd * 2 + m * nh * hd + y), "flops": 4.0 * pairs * nh * hd}


def exact(case, seed):
    """The results in 64 bits, from the definitions, a sequence at a time."""
    s = prepare(case, seed)
    news, lens = _lengths(case, seed)
    nh, nkv, hd, ps, m = case["nh"], case["nkv"], case["hd"], case["ps"], s["m"]
    pages = [s["table"][i, :-(-n // ps)].long() for i, n in enumerate(lens)]
    if case["op"] == "append":
        return _exact_append(case, s, news, lens, pages)
    q = (_rows(s["q"], m, nh * hd) if case["layout"] == "tiles" else s["q"]).reshape(m, nh, hd).double() * s["q_scale"]
    o = torch.zeros((m, nh, hd), dtype=torch.float64, device=q.device)
    first = 0
    for n, t, page in zip(news, lens, pages):
        rows, first = slice(first, first + n), first + n
        if t == 0:
            continue
        place = torch.arange(t, device=q.device)
        for h in range(nkv):
            keys = s["cache"][page, 0, h].reshape(-1, hd)[:t].double() * s["k_scale"]
            groups = s["cache"][page, 1, h].reshape(-1, hd, 16)
            values = groups[place // 16, :, place % 16].double() * s["v_scale"]
            for a in range(h * (nh // nkv), (h + 1) * (nh // nkv)):
                z = (q[rows, a] @ keys.t()) / math.sqrt(hd)
                if case["causal"]:
                    z = z.masked_fill(place[None, :] > (t - n + torch.arange(n, device=q.device))[:, None], -math.inf)
                o[rows, a] = torch.softmax(z, dim=1) @ values
    o = o.reshape(m, nh * hd)
    if case["kind"] == "i8":
        o = torch.round(o / s["out_scale"]).clamp(-127, 127) * s["out_scale"]
        o = _tiles(o) if _whole(case, m) else o
    return {"y": o}


def _exact_append(case, s, news, lens, pages):
    nh, nkv, hd, ps, m, rot = case["nh"], case["nkv"], case["hd"], case["ps"], s["m"], case["rot"]
    cols = (nh + 2 * nkv) * hd
    x = _rows(s["x"], m, cols) if case["x"] == "i8" and case["layout"] == "tiles" else s["x"]
    x = x.reshape(m, nh + 2 * nkv, hd).double() * s["x_scale"]
    store = s["cache"].double()
    q = torch.empty((m, nh, hd), dtype=torch.float64, device=x.device)
    rounded = lambda v, scale: torch.round(v / scale).clamp(-127, 127)  # noqa: E731
    first = 0
    for n, t, page in zip(news, lens, pages):
        part = x[first:first + n]
        place = torch.arange(t - n, t, device=x.device)
        if rot:
            turn = torch.polar(torch.full((n, rot // 2), s["factor"], dtype=torch.float64, device=x.device),
                               torch.outer((place + case["far"]).double(), s["freq"].double()))[:, None]
            pairs = part[:, :nh + nkv, :rot]
            if case["rope"] == "half":
                z = torch.complex(*(p.contiguous() for p in pairs.chunk(2, 2))) * turn
                part[:, :nh + nkv, :rot] = torch.cat([z.real, z.imag], 2)
            else:
                z = torch.view_as_complex(pairs.reshape(n, nh + nkv, rot // 2, 2).contiguous()) * turn
                part[:, :nh + nkv, :rot] = torch.view_as_real(z).reshape(n, nh + nkv, rot)
        q[first:first + n] = rounded(part[:, :nh], s["q_scale"])
        first += n
        if t == 0:
            continue
        for h in range(nkv):
            store[page[place // ps], 0, h, place % ps] = rounded(part[:, nh + h], s["k_scale"])
            groups = store[:, 1, h].reshape(-1, ps // 16, hd, 16)  # (a copy)
            groups[page[place // ps], place % ps // 16, :, place % 16] = rounded(part[:, nh + nkv + h], s["v_scale"])
            store[:, 1, h] = groups.reshape(-1, ps, hd)
    q = q.reshape(m, nh * hd) * s["q_scale"]
    store[:, 0] *= s["k_scale"]
    store[:, 1] *= s["v_scale"]
    return {"q": _tiles(q) if _whole(case, m) else q, "cache": store}
