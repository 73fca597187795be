"""Argument checks of cache_append and cache_attention: what the C ABI refuses, on the CPU (a refusal comes before any
launch), and the argument structs against a C compiler's."""
import os
import re
import struct
import subprocess

import pytest

import paper_2211_07715_amd as sl

INVALID, SHAPE, UNSUPPORTED = -1, -2, -5
P = 0x10000  # stands for a device address; refusals never read it
NAN, INF = float("nan"), float("inf")

APPEND = dict(x=P, m_tokens=8, seq_start=P, kv_len=P, page_table=P, positions=0, inv_freq=P, cache=P, q=P, n_seq=2,
              max_new=4, max_pages=3, n_pages=9, page_size=16, x_type=2, x_layout=0, n_heads=4, n_kv_heads=2, head_dim=64,
              rope_kind=1, rope_dim=64, q_layout=0, x_scale=0.1, rope_factor=1.0, q_scale=0.1, k_scale=0.1, v_scale=0.1)
ATTEND = dict(q=P, m_tokens=8, seq_start=P, kv_len=P, page_table=P, cache=P, y=P, workspace=P, workspace_bytes=1 << 40,
              n_seq=2, max_new=4, max_len=2048, max_pages=128, n_pages=300, page_size=16, q_layout=0, q_cols=256,
              n_heads=4, n_kv_heads=2, head_dim=64, causal=1, kind=3, y_layout=0, q_scale=0.1, k_scale=0.1, v_scale=0.1,
              softmax_scale=0.1, out_scale=0.1)


def append(**change):
    return sl.load().cache_append(sl._APPEND_ARGS.pack(*{**APPEND, **change}.values()), None)


def attend(**change):
    return sl.load().cache_attention(sl._CACHE_ARGS.pack(*{**ATTEND, **change}.values()), None)


def workspace(**change):
    return sl.load().cache_attention_workspace(sl._CACHE_ARGS.pack(*{**ATTEND, **change}.values()))


@pytest.mark.parametrize("change,status", [
    (dict(m_tokens=-1), SHAPE), (dict(m_tokens=2 ** 31), SHAPE), (dict(n_heads=3), SHAPE), (dict(n_heads=-2), SHAPE),
    (dict(n_kv_heads=0), SHAPE), (dict(head_dim=8), SHAPE), (dict(head_dim=144), SHAPE), (dict(head_dim=72), SHAPE),
    (dict(n_heads=2 ** 30, n_kv_heads=2 ** 30), SHAPE), (dict(n_seq=-1), SHAPE), (dict(max_new=-1), SHAPE),
    (dict(max_new=2 ** 31 - 1), SHAPE), (dict(max_pages=-1), SHAPE), (dict(n_pages=-1), SHAPE),
    (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE), (dict(page_size=512), SHAPE), (dict(page_size=0), SHAPE),
    (dict(max_pages=2 ** 27), SHAPE), (dict(q_scale=0.0), INVALID), (dict(k_scale=NAN), INVALID),
    (dict(v_scale=INF), INVALID), (dict(seq_start=0), INVALID), (dict(kv_len=0), INVALID), (dict(page_table=0), INVALID),
    (dict(cache=0), INVALID), (dict(kv_len=P + 2), INVALID), (dict(seq_start=P + 1), INVALID),
    (dict(page_table=P + 2), INVALID), (dict(cache=P + 8), INVALID)])
def test_both_refuse(change, status):
    assert append(**change) == status
    assert sl.load().sl_last_error() != b""
    assert attend(**change) == status
    assert sl.load().sl_last_error() != b""


@pytest.mark.parametrize("change,status", [
    (dict(x_type=0), INVALID), (dict(x_type=3), INVALID), (dict(x_layout=2), INVALID), (dict(x_scale=0.0), INVALID),
    (dict(x_scale=NAN), INVALID), (dict(rope_kind=3), INVALID), (dict(rope_kind=-1), INVALID), (dict(rope_dim=0), SHAPE),
    (dict(rope_dim=66), SHAPE), (dict(rope_dim=31), SHAPE), (dict(rope_factor=INF), INVALID), (dict(q_layout=2), INVALID),
    (dict(x=0), INVALID), (dict(x=P + 4), INVALID), (dict(q=P + 4), INVALID), (dict(inv_freq=0), INVALID),
    (dict(inv_freq=P + 2), INVALID), (dict(positions=P + 2), INVALID)])
def test_append_refuses(change, status):
    assert append(**change) == status
    assert sl.load().sl_last_error() != b""


@pytest.mark.parametrize("change,status", [
    (dict(n_heads=0), SHAPE), (dict(max_len=-1), SHAPE), (dict(max_len=2 ** 31 - 1), SHAPE), (dict(q_layout=-1), INVALID),
    (dict(q_cols=255), SHAPE), (dict(q_cols=264), SHAPE), (dict(q_cols=2 ** 24 + 16), SHAPE), (dict(causal=2), INVALID),
    (dict(kind=0), INVALID), (dict(kind=2), INVALID), (dict(y_layout=2), INVALID), (dict(kind=1, y_layout=1), INVALID),
    (dict(softmax_scale=0.0), INVALID), (dict(q_scale=1e20, k_scale=1e20), INVALID), (dict(out_scale=-1.0), INVALID),
    (dict(q=0), INVALID), (dict(y=0), INVALID), (dict(q=P + 8), INVALID), (dict(y=P + 8), INVALID),
    (dict(workspace=0), INVALID), (dict(workspace=P + 8), INVALID), (dict(workspace_bytes=0), INVALID)])
def test_attention_refuses(change, status):
    assert attend(**change) == status
    assert sl.load().sl_last_error() != b""


def test_more_than_a_launch_takes():
    big = dict(m_tokens=2 ** 31 - 256, n_seq=2 ** 31 - 1, max_new=2 ** 31 - 256)
    assert append(**big) == UNSUPPORTED
    assert attend(**big, workspace=0, workspace_bytes=0) == UNSUPPORTED
    assert workspace(**big) == 0


def test_null_args_and_nothing_to_do():
    lib = sl.load()
    assert lib.cache_append(None, None) == lib.cache_attention(None, None) == INVALID
    assert lib.cache_attention_workspace(None) == 0
    for change in (dict(m_tokens=0), dict(n_seq=0), dict(max_new=0)):
        none = dict(seq_start=0, kv_len=0, page_table=0, cache=0, q=0)
        assert append(x=0, inv_freq=0, **none, **change) == 0
        assert attend(y=0, workspace=0, workspace_bytes=0, **none, **change) == 0
        assert workspace(**change) == 0
        assert append(head_dim=8, **change) == attend(head_dim=8, **change) == SHAPE


def test_workspace_is_what_is_asked_for():
    need = workspace()
    assert need > 0 and need % 16 == 0
    assert attend(workspace_bytes=need - 1) == INVALID
    assert workspace(head_dim=7) == workspace(page_size=3) == 0
    assert workspace(n_seq=4096) == 0  # (enough sequences: no keys are split)


def test_shape_of_a_cache():
    assert sl.cache_shape(7, 32, 4, 96) == (7, 2, 4, 32, 96)


def test_argument_structs_match_the_header(tmp_path):
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    text = open(os.path.join(inc, "sparse_linear.h")).read()
    for name, fields, packed in (("sl_cache_append_args", APPEND, sl._APPEND_ARGS),
                                 ("sl_cache_attention_args", ATTEND, sl._CACHE_ARGS)):
        declared = re.findall(r"(\w+);", re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1))
        assert declared == list(fields)
        src = tmp_path / (name + ".c")
        src.write_text('#include "sparse_linear.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void){printf("%zu",'
                       f"sizeof({name}));" + "".join(f'printf(" %zu",offsetof({name},{f}));' for f in declared) +
                       "return 0;}\n")
        exe = str(tmp_path / name)
        subprocess.run(["gcc", "-I", inc, str(src), "-o", exe], check=True)
        size, *offsets = map(int, subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split())
        assert packed.size == size
        codes = [c for n, c in re.findall(r"(\d*)([a-zA-Z])", packed.format) for _ in range(int(n or 1) if n != "0" else 0)]
        assert [struct.calcsize("".join(codes[:i]) + "0" + codes[i]) for i in range(len(codes))] == offsets
