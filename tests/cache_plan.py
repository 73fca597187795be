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
Attention = namedtuple("Attention", "prompt by_length fits tile_rows splits split_keys tiles")


@functools.lru_cache(None)
def _program(text):
    where = tempfile.mkdtemp()
    src, exe = os.path.join(where, "plan.cpp"), os.path.join(where, "plan")
    with open(src, "w") as f:
        f.write(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", CSRC, src, "-o", exe], check=True)
    return exe


def attention(m_tokens, n_seq, max_new, max_len, n_heads, n_kv_heads, head_dim, causal=True):
    given = (m_tokens, n_seq, max_new, max_len, n_heads, n_kv_heads, head_dim, int(causal))
    out = subprocess.run([_program(PROGRAM)], input=" ".join(map(str, given)), check=True, stdout=subprocess.PIPE, text=True)
    return Attention(*map(int, out.stdout.split()))
