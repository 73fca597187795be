// What the kernels of a decoder's cache share (gfx950). Not part of the public ABI.
#pragma once

#include "attention_device.h"
#include "cache_plan.h"

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
    int32_t by_length;  // tiles in order of the keys that they see
    float c2, k2, vs, unit, inv_group;
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

// v of a lane and those before it: their sum, or the largest.
template <class F>
__device__ __forceinline__ int32_t running(int32_t v, int32_t none, F with)
{
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x111, 0xf, 0xf, false));  // 1, 2, 4, 8 lanes before in 16
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x112, 0xf, 0xf, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x114, 0xf, 0xf, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x118, 0xf, 0xf, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x142, 0xa, 0xf, false));  // lanes 15 and 47 to the 16 after them
    return with(v, __builtin_amdgcn_update_dpp(none, v, 0x143, 0xc, 0xf, false));  // lane 31 to the last 32
}
__device__ __forceinline__ int32_t running_sum(int32_t v)
{
    return running(v, 0, [](int32_t x, int32_t y) { return x + y; });
}
__device__ __forceinline__ int32_t lanes_sum(int32_t v) { return __builtin_amdgcn_readlane(running_sum(v), 63); }
__device__ __forceinline__ int32_t lanes_max(int32_t v)  // (of numbers that are not below 0)
{
    return __builtin_amdgcn_readlane(running(v, 0, [](int32_t x, int32_t y) { return max(x, y); }), 63);
}

// The lengths of all sequences of a call that has few, up to S of them a lane.
template <int S>
struct Lengths {
    int32_t start[S], end[S], len[S];
    __device__ __forceinline__ Lengths(const CacheArgs &a, int32_t lane)
    {
#pragma unroll
        for (int g = 0; g < S; ++g) {
            const int32_t seq = 64 * g + lane;
            start[g] = end[g] = len[g] = 0;
            if (64 * g < a.n_seq && seq < a.n_seq) {
                start[g] = a.seq_start[seq];
                end[g] = a.seq_start[seq + 1];
                len[g] = a.kv_len[seq];
            }
        }
    }
    __device__ __forceinline__ int32_t keys(const CacheArgs &a, int g) const
    {
        return (int32_t)min((int64_t)max(len[g], 0), (int64_t)a.max_pages << a.shift);
    }
    __device__ __forceinline__ bool equal(const CacheArgs &a, int32_t lane) const  // all sequences' are
    {
        const int32_t n0 = __builtin_amdgcn_readfirstlane(tokens_between(start[0], end[0], a.m).n);
        const int32_t k0 = __builtin_amdgcn_readfirstlane(keys(a, 0));
        bool same = true;
#pragma unroll
        for (int g = 0; g < S; ++g)
            same = same && (64 * g + lane >= a.n_seq || (tokens_between(start[g], end[g], a.m).n == n0 && keys(a, g) == k0));
        return __all(same);
    }
};

struct Place {
    int32_t seq, from_last, start, end, len;  // a tile's sequence (-1: none), its number from the last, the lengths
};
// Tile `nth` of all sequences', those that see the most keys first. A sequence's last tile's level says by how many
// tiles' tokens it is shorter than the longest, tile j before that is on the jth level after it (without `causal` on the
// same). How many tiles lie above a level is a sum over lanes, so tile nth's level is found by halves.
template <int S>
__device__ __forceinline__ Place nth_longest(const CacheArgs &a, const Lengths<S> &of, int32_t nth, int32_t tile_rows)
{
    int32_t tiles[S], level[S], longest = 0, all = 0, last = 0;
#pragma unroll
    for (int g = 0; g < S; ++g) {
        const int64_t rows = (int64_t)tokens_between(of.start[g], of.end[g], a.m).n * a.group;
        tiles[g] = (int32_t)min((rows + tile_rows - 1) / tile_rows, (int64_t)a.tiles);
        longest = max(longest, of.keys(a, g));
    }
    longest = lanes_max(longest);
#pragma unroll
    for (int g = 0; g < S; ++g) {
        level[g] = (int32_t)((uint32_t)(longest - of.keys(a, g)) / (uint32_t)max(tile_rows / a.group, 1));
        all += tiles[g];
        last = max(last, level[g] + tiles[g]);
    }
    const auto above = [&](int32_t l, int g) {
        return a.causal ? min(max(l - level[g], 0), tiles[g]) : l > level[g] ? tiles[g] : 0;
    };
    const auto all_above = [&](int32_t l) {
        int32_t sum = 0;
#pragma unroll
        for (int g = 0; g < S; ++g) sum += above(l, g);
        return lanes_sum(sum);
    };
    Place at{-1, 0, 0, 0, 0};
    if (nth >= lanes_sum(all)) return at;
    int32_t lo = 0, hi = lanes_max(last);
    while (hi - lo > 1) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (all_above(mid) <= nth)
            lo = mid;
        else
            hi = mid;
    }
    int32_t rest = nth - all_above(lo);
#pragma unroll
    for (int g = 0; g < S; ++g) {
        if (at.seq >= 0 || 64 * g >= a.n_seq) continue;
        const int32_t mine = above(lo + 1, g) - above(lo, g), sum = running_sum(mine), before = sum - mine;
        const uint64_t found = __ballot(before <= rest && rest < sum);
        if (!found) {
            rest -= __builtin_amdgcn_readlane(sum, 63);
            continue;
        }
        const int k = __builtin_ctzll(found);
        const int32_t its_level = __builtin_amdgcn_readlane(level[g], k), its_first = __builtin_amdgcn_readlane(before, k);
        at.seq = 64 * g + k;
        at.from_last = a.causal ? lo - its_level : rest - its_first;
        at.start = __builtin_amdgcn_readlane(of.start[g], k);
        at.end = __builtin_amdgcn_readlane(of.end[g], k);
        at.len = __builtin_amdgcn_readlane(of.len[g], k);
    }
    return at;
}

// floats of a part's record in the workspace: m, l and O of a workgroup's rows
__host__ __device__ constexpr int64_t record(int hd, int rows) { return rows * (int64_t)(hd + 2); }

}  // namespace sl
