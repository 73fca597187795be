"""What calls of a decoder's cache launch (csrc/cache_plan.h), from a CPU build of it."""
import functools
import os
import subprocess
import tempfile
from collections import namedtuple

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2211_07715_amd", "csrc")

PROGRAM = r"""
#include <stdio.h>
#include "cache_plan.h"
using namespace sl;
int main()
{
    sl_cache_attention_args a{};
    while (scanf("%ld %d %d %d %d %d %d %d", &a.m_tokens, &a.n_seq, &a.max_new, &a.max_len, &a.n_heads, &a.n_kv_heads,
                 &a.head_dim, &a.causal) == 8) {
        const AttentionPlan p = plan_of(a);
        printf("%d %d %d %d %d %d %d\n", p.prompt, p.by_length, p.fits, p.tile_rows, p.splits, p.split_keys, p.tiles);
    }
}
"""
APPEND = r"""
#include <stdio.h>
#include "cache_plan.h"
using namespace sl;
int main()
{
    static int8_t some;
    int queries;
    sl_cache_append_args a{};
    while (scanf("%ld %d %d %d %d %d %d %d %d", &a.m_tokens, &a.n_seq, &a.max_new, &a.n_heads, &a.n_kv_heads, &a.head_dim,
                 &a.rope_kind, &a.rope_dim, &queries) == 9) {
        a.q = queries ? &some : nullptr;
        const AppendPlan p = plan_of(a);
        printf("%d %d %d %d %d %d %d %d %d %d %d %d\n", p.fits, p.step, p.vec, p.groups, p.q_columns, p.k_columns, p.v_columns,
               p.q_parts, p.k_parts, p.parts, p.per, p.v_per);
    }
}
"""
Append = namedtuple("Append", "fits step vec groups q_columns k_columns v_columns q_parts k_parts parts per v_per")
Attention = namedtuple("Attention", "prompt by_length fits tile_rows splits split_keys tiles")


@functools.lru_cache(None)
def _program(text):
    where = tempfile.mkdtemp()
    src, exe = os.path.join(where, "plan.cpp"), os.path.join(where, "plan")
    with open(src, "w") as f:
        f.write(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", CSRC, src, "-o", exe], check=True)
    return exe


def _run(program, given):
    return map(int, subprocess.run([_program(program)], input=" ".join(map(str, given)), check=True, stdout=subprocess.PIPE,
                                   text=True).stdout.split())


def attention(m_tokens, n_seq, max_new, max_len, n_heads, n_kv_heads, head_dim, causal=True):
    return Attention(*_run(PROGRAM, (m_tokens, n_seq, max_new, max_len, n_heads, n_kv_heads, head_dim, int(causal))))


def append(m_tokens, n_seq, max_new, n_heads, n_kv_heads, head_dim, rope_kind=0, rope_dim=0, queries=True):
    return Append(*_run(APPEND, (m_tokens, n_seq, max_new, n_heads, n_kv_heads, head_dim, rope_kind, rope_dim, int(queries))))
