"""GPU tests of what attention_run and attention_select do with sizes at and past
their ranges: starts and key lengths that are brought in, nothing to do, and launches
of more work than one takes."""
import numpy as np
import pytest

import attention_bars as bars
import encoder_ref as ref

pytestmark = pytest.mark.gpu
T = 1  # LAYOUT_T16X32


def _i32(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def test_sizes_that_are_none(hip):
    """Refused by name: by the binding where it makes a shape or a scale of them, otherwise by the library."""
    import torch
    x = torch.zeros((64, 3 * 64), dtype=torch.int8, device="cuda")
    start = _i32([0, 64])
    lists = torch.zeros((1, 1, 1, 1), dtype=torch.int32, device="cuda")
    for qb in (0, -64):
        with pytest.raises(ValueError):
            hip.attention(x, 0.04, start, 64, 1, 64, kind=1, blocks=lists, query_block=qb)
        with pytest.raises(ValueError):
            hip.select_blocks(x, start, 64, 1, 64, 1, query_block=qb)
    none = torch.zeros((64, 0), dtype=torch.int8, device="cuda")
    for nh, hd, nkv, t, error in ((1, 0, 1, none, ValueError), (-1, -64, -1, x, ValueError), (1, -64, -2, x, ValueError),
                                  (0, 64, 0, none, hip.SparseLinearError), (3, 64, 0, x, hip.SparseLinearError)):
        with pytest.raises(error):
            hip.attention(t, 0.04, start, 64, nh, hd, n_kv_heads=nkv, kind=1)
        with pytest.raises(error):
            hip.select_blocks(t, start, 64, nh, hd, 1, n_kv_heads=nkv)
    with pytest.raises(ValueError):
        hip.select_blocks(x, start, -64, 1, 64, 1)
    with pytest.raises(ValueError):
        hip.attention(x, 0.04, start, -64, 1, 64, blocks=lists)
    with pytest.raises(hip.SparseLinearError):
        hip.attention(x, 0.04, start, -64, 1, 64)


def test_no_tokens(hip):
    """An empty batch of sequences is nothing to do with lists as without them; the lists name no block."""
    import torch
    for layout in (0, T):
        x = torch.empty(hip.t16x32_shape(0, 192) if layout == T else (0, 192), dtype=torch.int8, device="cuda")
        args = dict(x_layout=layout, m_tokens=0)
        out = torch.full((3, 1, 2, 4), 5, dtype=torch.int32, device="cuda")
        for blocks in (hip.select_blocks(x, _i32([0, 0, 0, 0]), 128, 1, 64, 4, **args),
                       hip.select_blocks(x, _i32([0, 0, 0, 0]), 128, 1, 64, 4, out=out, stream=torch.cuda.Stream(), **args)):
            torch.cuda.synchronize()
            assert blocks.shape == (3, 1, 2, 4) and (blocks == -1).all()
            y = hip.attention(x, 0.04, _i32([0, 0, 0, 0]), 128, 1, 64, kind=1, blocks=blocks, **args)
            assert y.shape == (0, 64)


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("layout", [0, T])
@pytest.mark.parametrize("given,keys,inside,inside_keys", [
    ([-5, 40, 1000], None, [0, 40, 150], None),
    ([-(2 ** 31), 2, 2 ** 31 - 1], None, [0, 2, 150], None),
    ([7, 90, 5000], [-3, 1000], [7, 90, 150], [0, 60]),
    ([-1, 65, 150], [2 ** 31 - 1, -(2 ** 31)], [0, 65, 150], [65, 0]),
    ([300, 400, 500], None, [150, 150, 150], None)])
def test_starts_and_key_lengths_are_brought_in(hip, given, keys, inside, inside_keys, layout, kind):
    """Every token of every sequence as with the numbers that they are brought to; tokens of none stay as they are."""
    import torch
    m, nh, hd = 150, 2, 64
    x = bars.codes(np.random.default_rng(1), m, 3 * nh * hd)
    xd = torch.from_numpy(np.ascontiguousarray(hip.to_t16x32(x, fill=99) if layout == T else x)).cuda()

    def both(starts, key_len):
        start, kl = _i32(starts), None if key_len is None else _i32(key_len)
        args = dict(key_len=kl, x_layout=layout, m_tokens=m)
        blocks = hip.select_blocks(xd, start, m, nh, hd, 2, **args)
        out = []
        for lists in (None, blocks):
            y = torch.full((m, nh * hd), 77, dtype=torch.float32 if kind == 1 else torch.int8, device="cuda")
            out.append(hip.attention(xd, 0.04, start, m, nh, hd, kind=kind, out_scale=0.02, blocks=lists, out=y, **args))
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in (blocks, *out)]

    got, want = both(given, keys), both(inside, inside_keys)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)
    assert np.array_equal(got[0], ref.select(x, np.array(inside), nh, nh, hd, 2, m, 64, inside_keys))
    y, bar = bars.attention(x, float(np.float32(0.04)), np.array(inside), nh, nh, hd, hd ** -0.5, inside_keys)
    first, last = inside[0], inside[-1]
    so = float(np.float32(0.02)) if kind == 3 else None
    bars.assert_within(got[1][first:last], y[first:last], bar[first:last], so)
    assert (got[1][:first] == 77).all() and (got[1][last:] == 77).all()


def _select(hip, x, start, nh, nkv, hd, top_k, max_len, qb):
    import torch
    print(f"select {len(start) - 1} sequences to {max_len}, heads {nh}/{nkv}x{hd}, query_block {qb}", flush=True)
    out = hip.select_blocks(torch.from_numpy(x).cuda(), _i32(start.tolist()), max_len, nh, hd, top_k, n_kv_heads=nkv,
                            query_block=qb)
    torch.cuda.synchronize()
    return out


def test_select_of_many_sequences(hip):
    """More sequences than a launch has a dimension for."""
    rng = np.random.default_rng(3)
    lens = np.minimum(rng.geometric(0.96, 70000) - 1, 5)
    lens[[5, 65535, 65536, 69999]] = 150, 140, 200, 131
    x = bars.codes(rng, int(lens.sum()), 3 * 16)
    start = bars.starts(lens)
    got = _select(hip, x, start, 1, 1, 16, 2, 200, 64).cpu().numpy()
    assert np.array_equal(got, ref.select(x, start, 1, 1, 16, 2, 200, 64))


def test_select_of_many_heads(hip):
    rng = np.random.default_rng(4)
    lens, nh = [40, 150], 66000
    x = bars.codes(rng, sum(lens), (nh + 4) * 16)
    start = bars.starts(lens)
    got = _select(hip, x, start, nh, 2, 16, 2, 150, 64).cpu().numpy()
    assert np.array_equal(got, ref.select(x, start, nh, 2, 16, 2, 150, 64))


@pytest.mark.parametrize("nh,n_seq,max_len,qb", [(1024, 66, 8192, 16), (1, 2100, 262144, 128), (2048, 66, 8192, 16)])
def test_select_of_more_than_a_launch(hip, nh, n_seq, max_len, qb):
    """Lists, or blocks of keys, of 2^31 and 2^32 threads and more; nearly all of sequences much shorter than max_len."""
    import torch
    rng = np.random.default_rng(n_seq)
    lens = [1] * n_seq
    lens[0], lens[7], lens[-1] = 150, 200, 131
    x = bars.codes(rng, sum(lens), (nh + 2) * 16)
    start = bars.starts(lens)
    got = _select(hip, x, start, nh, 1, 16, 1, max_len, qb)
    for s in (0, 1, 7, n_seq - 2, n_seq - 1):
        want = ref.select(x[start[s]:start[s + 1]], np.array([0, lens[s]]), nh, 1, 16, 1, max(lens), qb)[0]
        assert np.array_equal(got[s, :, :want.shape[1]].cpu().numpy(), want)
        got[s, :, :want.shape[1]] = -1
    got[:, :, 0] = torch.where(got[:, :, 0] == 0, -1, got[:, :, 0])  # (a sequence of one token has its one block)
    assert bool((got == -1).all())
