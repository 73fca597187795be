"""64-bit definitions of cache_append and cache_attention on the host (numpy), written from the formulas, a token at a
time, and the pages of a cache taken apart."""
import numpy as np

NONE, HALF, INTERLEAVED = 0, 1, 2


def slots_of(page_table, page_size, n_pages, seq, count):
    """(page, place) of a sequence's first `count` slots; page -1 where the table names none."""
    out = []
    for p in range(count):
        e = p // page_size
        page = int(page_table[seq, e]) if e < page_table.shape[1] else -1
        out.append((page if 0 <= page < n_pages else -1, p % page_size))
    return out


def key_of(cache, page, head, place):
    return cache[page, 0, head, place]


def value_of(cache, page, head, place):
    """A view of the [head_dim] values of one slot: 16 slots' codes of a feature lie together."""
    _, _, _, ps, hd = cache.shape
    return cache[page, 1, head].reshape(ps // 16, hd, 16)[place // 16, :, place % 16]


def rotate(x, pos, kind, inv_freq, factor):
    """x [heads, head_dim] in 64 bits."""
    if kind == NONE:
        return x
    y = x.copy()
    half = len(inv_freq)
    w = float(pos) * inv_freq.astype(np.float64)
    c, s = factor * np.cos(w), factor * np.sin(w)
    a, b = (slice(0, half), slice(half, 2 * half)) if kind == HALF else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
    return y


def append(x, seq_start, kv_len, page_table, page_size, n_pages, nh, nkv, hd, kind, inv_freq, factor, positions=None):
    """x [M, cols] values in 64 bits. Returns (queries {token: [nh, hd]}, [(page, place, keys, values)]), unrounded."""
    queries, stored = {}, []
    for s in range(len(kv_len)):
        first, end = int(seq_start[s]), int(seq_start[s + 1])
        length = max(int(kv_len[s]), 0)
        where = slots_of(page_table, page_size, n_pages, s, length)
        for t in range(first, end):
            slot = length - (end - first) + (t - first)
            pos = slot if positions is None else int(positions[t])
            row = x[t].reshape(nh + 2 * nkv, hd)
            qk = rotate(row[:nh + nkv], pos, kind, inv_freq, factor)
            queries[t] = qk[:nh]
            if slot >= 0 and where[slot][0] >= 0:
                stored.append((*where[slot], qk[nh:], row[nh + nkv:]))
    return queries, stored


def attention(q, cache, seq_start, kv_len, page_table, nh, scale, causal):
    """q [M, >= nh * hd] codes, scale = q_scale k_scale softmax_scale. Returns ({token: [nh, hd]}: the mean of the
    values' codes under the softmax weights, most keys that a token saw)."""
    n_pages, _, nkv, ps, hd = cache.shape
    out, most = {}, 0
    for s in range(len(kv_len)):
        first, end = int(seq_start[s]), int(seq_start[s + 1])
        length = max(int(kv_len[s]), 0)
        where = [(i, w) for i, w in enumerate(slots_of(page_table, ps, n_pages, s, length)) if w[0] >= 0]
        at = np.array([i for i, _ in where], dtype=np.int64)
        page = np.array([w[0] for _, w in where], dtype=np.int64)
        place = np.array([w[1] for _, w in where], dtype=np.int64)
        keys = cache[page, 0, :, place].astype(np.float64).transpose(1, 0, 2)  # [nkv, keys, hd]
        groups = cache[:, 1].reshape(n_pages, nkv, ps // 16, hd, 16)
        values = groups[page, :, place // 16, :, place % 16].astype(np.float64).transpose(1, 0, 2)
        for t in range(first, end):
            last = length - (end - first) + (t - first) if causal else length - 1
            seen = at <= last
            y = np.zeros((nh, hd))
            if seen.any():
                most = max(most, int(seen.sum()))
                rows = q[t, :nh * hd].reshape(nkv, nh // nkv, hd).astype(np.float64)
                z = rows @ keys[:, seen].transpose(0, 2, 1) * scale
                w = np.exp(z - z.max(2, keepdims=True))
                y = ((w / w.sum(2, keepdims=True)) @ values[:, seen]).reshape(nh, hd)
            out[t] = y
    return out, most
