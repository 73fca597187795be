// What the kernels of a decoder's cache share (gfx950). Not part of the public ABI.
#pragma once

#include "attention_device.h"

namespace sl {

// tokens first .. first + n - 1 of a call that belong to a sequence
struct Tokens {
    int32_t first, n;
};
__device__ __forceinline__ Tokens tokens_of(const int32_t *seq_start, int32_t s, int64_t m)
{
    const int32_t m32 = (int32_t)m;
    const int32_t b = min(max(seq_start[s], 0), m32);
    return {b, min(max(seq_start[s + 1], b), m32) - b};
}

// cache_attention's arguments as its kernels take them
struct CacheArgs {
    const int8_t *q, *cache;
    const int32_t *seq_start, *kv_len, *page_table;
    void *y;
    float *work;
    int64_t m;
    int32_t n_seq, tiles, splits, split_keys;
    int32_t n_heads, n_kv, group, hd, q_cols, q_cb, y_cb, shift, max_pages, n_pages, causal, y_f32, join_rows, seq0;
    float c2, k2, vs, inv_so, inv_group;
};

// cache_attention for many queries a sequence (kernels_cache_prompt.hip)
sl_status launch_cache_prompt(CacheArgs a, const sl_cache_attention_args &args, hipStream_t s);

}  // namespace sl
