// What the kernels of a decoder's cache share (gfx950). Not part of the public ABI.
#pragma once

#include "attention_device.h"

namespace sl {

// tokens first .. first + n - 1 of a call that belong to a sequence
struct Tokens {
    int32_t first, n;
};
__device__ __forceinline__ Tokens tokens_between(int32_t start, int32_t end, int64_t m)
{
    const int32_t m32 = (int32_t)m;
    const int32_t b = min(max(start, 0), m32);
    return {b, min(max(end, b), m32) - b};
}
__device__ __forceinline__ Tokens tokens_of(const int32_t *seq_start, int32_t s, int64_t m)
{
    return tokens_between(seq_start[s], seq_start[s + 1], m);
}
typedef const __attribute__((address_space(4))) int32_t *ScalarTable;  // read through the scalar cache

// cache_attention's arguments as its kernels take them
struct CacheArgs {
    const int8_t *q, *cache;
    const int32_t *seq_start, *kv_len, *page_table;
    void *y;
    float *work;
    int64_t m;
    int32_t n_seq, tiles, splits, split_keys;
    int32_t n_heads, n_kv, group, hd, q_cols, q_cb, y_cb, shift, max_pages, n_pages, causal, y_f32, tile_rows, join_group, seq0, group_shift;
    int32_t by_length;  // tiles of prompts in order of the keys that they see
    float c2, k2, vs, inv_so, inv_group;
};

// cache_attention for many queries a sequence (kernels_cache_prompt.hip): tile_rows, 64 or 128, (query, head) pairs a
// workgroup (64 for heads to 64 features only)
sl_status launch_cache_prompt(const CacheArgs &a, dim3 grid, hipStream_t s);

// token of a (query, head) row of a key head: x / group
__device__ __forceinline__ int64_t by_group(const CacheArgs &a, int64_t x)
{
    return a.group_shift >= 0 ? x >> a.group_shift : x < 0x7fffffff ? (int64_t)((uint32_t)x / (uint32_t)a.group) : x / a.group;
}
__device__ __forceinline__ uint32_t by_group(const CacheArgs &a, uint32_t x)
{
    return a.group_shift >= 0 ? x >> a.group_shift : x / (uint32_t)a.group;
}

// floats of a part's record in the workspace: m, l and O of a workgroup's rows
__host__ __device__ constexpr int64_t record(int hd, int rows) { return rows * (int64_t)(hd + 2); }

}  // namespace sl
