"""Plain numpy definitions, in 64 bits, of the operators between the linears,
for the tests to compare with. They share no code with the library."""
import numpy as np

BLOCK = 64


def norm_rows(x, kind, gamma, beta, eps):
    """kind 0: as it is, 1: LayerNorm, 2: RMS."""
    if kind == 0:
        return x
    mean = x.mean(1, keepdims=True) if kind == 1 else 0.0
    x = (x - mean) / np.sqrt(np.square(x - mean).mean(1, keepdims=True) + eps)
    if gamma is not None:
        x = x * gamma
    return x if beta is None else x + beta


def residual_norm(y, r, gate, rscale, post, pgamma, pbeta, kind, gamma, beta, eps):
    """(t, h, u), all float64 [rows, cols]."""
    t = norm_rows(y, post, pgamma, pbeta, eps)
    h = t if gate is None else t * gate
    if r is not None:
        h = rscale * r + h
    return t, h, norm_rows(h, kind, gamma, beta, eps)


def split_heads(x, start, s, nh, nkv, hd, key_len=None):
    """q [n, nh, hd], k and v [keys, nkv, hd] of sequence s, float64."""
    part = x[start[s]:start[s + 1]].reshape(-1, nh + 2 * nkv, hd).astype(np.float64)
    keys = len(part) if key_len is None else key_len[s]
    return part[:, :nh], part[:keys, nh:nh + nkv], part[:keys, nh + nkv:]


def attention(x, x_scale, start, nh, nkv, hd, softmax_scale, key_len=None, lists=None, query_block=64):
    """[M, nh * hd] float64 (zeros for tokens of no sequence), and the largest spread of a row's logits."""
    out, spread = np.zeros((len(x), nh, hd)), 0.0
    for s in range(len(start) - 1):
        q, k, v = split_heads(x, start, s, nh, nkv, hd, key_len)
        n, keys = len(q), len(k)
        if n == 0 or keys == 0:
            continue
        for h in range(nh):
            kv = h // (nh // nkv)
            z = q[:, h] @ k[:, kv].T * (float(x_scale) ** 2 * softmax_scale)
            if lists is not None:
                z = np.where(listed(lists[s, h], n, keys, query_block), z, -np.inf)
            some = np.isfinite(z).any(1)
            top = np.where(some, z.max(1), 0.0)
            low = np.where(np.isfinite(z), z, np.inf).min(1)
            spread = max(spread, float(np.max(np.where(some, top - low, 0.0))))
            p = np.exp(z - top[:, None])
            p = np.divide(p, p.sum(1, keepdims=True), out=np.zeros_like(p), where=some[:, None])
            out[start[s]:start[s + 1], h] = p @ v[:, kv] * x_scale
    return out.reshape(len(x), nh * hd), spread


def listed(lists, n, keys, query_block):
    """[n, keys]: key j is in a block that query i's list names."""
    blocks = -(-keys // BLOCK)
    use = np.zeros((len(lists), blocks), bool)
    for i, row in enumerate(lists):
        use[i, [b for b in row if 0 <= b < blocks]] = True
    qb = np.arange(n) // query_block
    rows = np.where((qb < len(lists))[:, None], use[np.minimum(qb, len(lists) - 1)], False)
    return rows[:, np.arange(keys) // BLOCK]


def select(x, start, nh, nkv, hd, top_k, max_len, query_block, key_len=None):
    """[n_seq, nh, ceil(max_len / query_block), top_k] int32, from whole-number scores."""
    n_seq = len(start) - 1
    out = np.full((n_seq, nh, -(-max_len // query_block), top_k), -1, np.int32)
    for s in range(n_seq):
        q, k, _ = split_heads(x.astype(np.int64), start, s, nh, nkv, hd, key_len)
        q, k = q.astype(np.int64), k.astype(np.int64)
        if len(q) == 0 or len(k) == 0:
            continue
        ks = []
        for b in range(0, len(k), BLOCK):
            part = k[b:b + BLOCK]
            total, n = 64 * part.sum(0), len(part)
            low, rest = total // n, total % n
            ks.append(low + ((2 * rest > n) | ((2 * rest == n) & (low % 2 == 1))))
        ks = np.stack(ks)  # [blocks, nkv, hd]
        for i in range(0, len(q), query_block):
            qs = q[i:i + query_block].sum(0)  # [nh, hd]
            for h in range(nh):
                score = ks[:, h // (nh // nkv)] @ qs[h]
                best = np.sort(np.argsort(-score, kind="stable")[:top_k])
                out[s, h, i // query_block, :len(best)] = best
    return out
