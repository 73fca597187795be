"""Argument checks of residual_norm, attention and select_blocks: what the C ABI
refuses, on the CPU (a refusal comes before any launch)."""
import struct

import pytest

import paper_2211_07715_amd as sl

INVALID, SHAPE, UNSUPPORTED = -1, -2, -5
P = 0x10000  # stands for a device address; refusals never read it

NORM = dict(rows=4, y=P, r=0, gate=0, post_gamma=0, post_beta=0, gamma=0, beta=0, h=0, u=0, q=P, cols=64, y_type=1,
            y_layout=0, r_type=0, r_layout=0, gate_kind=0, post_kind=0, norm_kind=1, q_layout=0, y_scale=1.0,
            r_scale=1.0, residual_scale=1.0, eps=1e-6, out_scale=0.1)
ATTN = dict(x=P, m_tokens=128, seq_start=P, key_len=0, blocks=0, y=P, n_seq=1, max_len=128, x_layout=0, n_heads=2,
            n_kv_heads=2, head_dim=64, top_k=4, query_block=64, kind=3, y_layout=0, x_scale=0.1, softmax_scale=0.1,
            out_scale=0.1)
NAN, INF = float("nan"), float("inf")


def norm(**change):
    return sl.load().residual_norm(sl._NORM_ARGS.pack(*{**NORM, **change}.values()), None)


def attn(**change):
    return sl.load().attention_run(sl._ATTN_ARGS.pack(*{**ATTN, **change}.values()), None)


def select(blocks=P, workspace=P, size=1 << 40, **change):
    return sl.load().attention_select(sl._ATTN_ARGS.pack(*{**ATTN, **change}.values()), blocks, workspace, size, None)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=65536), SHAPE), (dict(y_type=0), INVALID),
    (dict(y_type=3), INVALID), (dict(r_type=3), INVALID), (dict(r_type=-1), INVALID),
    (dict(y_type=2, y_layout=2), INVALID), (dict(r_type=2, r=P, r_layout=2), INVALID), (dict(q_layout=-1), INVALID),
    (dict(y_type=2, y_scale=0.0), INVALID), (dict(y_type=2, y_scale=NAN), INVALID),
    (dict(r_type=2, r=P, r_scale=-1.0), INVALID), (dict(out_scale=0.0), INVALID), (dict(out_scale=INF), INVALID),
    (dict(residual_scale=INF), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID),
    (dict(gate_kind=4), INVALID), (dict(gate_kind=1), INVALID), (dict(post_kind=3), INVALID),
    (dict(norm_kind=-1), INVALID), (dict(q=0), INVALID), (dict(y=0), INVALID), (dict(r_type=1), INVALID),
    (dict(y=P + 2), INVALID), (dict(gamma=P + 1), INVALID), (dict(h=P + 3), INVALID),
    (dict(y_type=2, y_layout=1, y=P + 4), INVALID), (dict(q_layout=1, q=P + 8), INVALID)])
def test_residual_norm_refuses(change, status):
    assert norm(**change) == status
    assert sl.load().sl_last_error() != b""


@pytest.mark.parametrize("change,status", [
    (dict(m_tokens=-1), SHAPE), (dict(m_tokens=2 ** 31), SHAPE), (dict(n_heads=3), SHAPE), (dict(n_heads=0), SHAPE),
    (dict(n_kv_heads=0), SHAPE), (dict(head_dim=8), SHAPE), (dict(head_dim=144), SHAPE), (dict(head_dim=72), SHAPE),
    (dict(n_heads=2 ** 30, n_kv_heads=2 ** 30), SHAPE), (dict(n_seq=-1), SHAPE), (dict(max_len=-1), SHAPE),
    (dict(x_layout=2), INVALID), (dict(x=0), INVALID), (dict(seq_start=0), INVALID), (dict(x=P + 4), INVALID),
    (dict(seq_start=P + 2), INVALID), (dict(key_len=P + 1), INVALID)])
def test_attention_and_select_refuse(change, status):
    assert attn(**change) == status
    assert select(**change) == status
    assert sl.load().sl_last_error() != b""


@pytest.mark.parametrize("change,status", [
    (dict(kind=0), INVALID), (dict(kind=2), INVALID), (dict(y_layout=3), INVALID), (dict(kind=1, y_layout=1), INVALID),
    (dict(x_scale=0.0), INVALID), (dict(softmax_scale=NAN), INVALID), (dict(x_scale=1e20), INVALID),
    (dict(out_scale=-1.0), INVALID), (dict(blocks=P, query_block=48), SHAPE), (dict(blocks=P, top_k=0), SHAPE),
    (dict(blocks=P + 2), INVALID), (dict(y=0), INVALID), (dict(y=P + 8), INVALID)])
def test_attention_refuses(change, status):
    assert attn(**change) == status


def test_select_refuses():
    assert select(query_block=0) == SHAPE
    assert select(top_k=0) == SHAPE
    assert select(max_len=262145) == UNSUPPORTED
    assert select(blocks=0) == INVALID
    assert select(workspace=0) == INVALID
    assert select(workspace=P + 8) == INVALID
    need = sl.load().attention_select_workspace(sl._ATTN_ARGS.pack(*ATTN.values()))
    assert need == (128 // 64 + 1 + 2) * 2 * 64 * 2
    assert select(size=need - 16) == INVALID
    assert sl.load().attention_select_workspace(None) == 0


def test_null_args_and_nothing_to_do():
    lib = sl.load()
    assert lib.residual_norm(None, None) == lib.attention_run(None, None) == INVALID
    assert lib.attention_select(None, None, None, 0, None) == INVALID
    assert norm(rows=0, y=0, q=P) == 0
    assert attn(m_tokens=0, x=0, y=0) == attn(n_seq=0, y=0) == attn(max_len=0, y=0) == 0
    assert select(n_seq=0, blocks=0, workspace=0) == select(max_len=0, blocks=0) == 0


def test_argument_structs_match_the_header(tmp_path):
    """The binding packs the structs by hand: sizes and every field's offset as a C compiler lays them out."""
    import os
    import re
    import subprocess
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    text = open(os.path.join(inc, "sparse_linear.h")).read()
    for name, fields, packed in (("sl_residual_norm_args", NORM, sl._NORM_ARGS), ("sl_attention_args", ATTN, sl._ATTN_ARGS)):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
        declared = re.findall(r"(\w+);", body)
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
