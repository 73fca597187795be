// What a call of cache_append or cache_attention launches: which kernel, how many workgroups, and what each of them has.
// Whole numbers of the arguments alone, for the host. Not part of the public ABI.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "../../include/sparse_linear.h"

namespace sl {

constexpr int kMostSorted = 256;                  // sequences that are taken in order of their lengths
constexpr int32_t kMostGrid = 65535;              // workgroups of a launch in its second and third dimension
constexpr int64_t kMostItems = 0x7fffffff / 256;  // and of a call, of 256 threads: under 2^31 threads

struct AttentionPlan {
    bool prompt, by_length, fits;  // (fits: else the call has more work items than a launch takes)
    int32_t tile_rows, splits, split_keys, tiles;
};

inline AttentionPlan plan_of(const sl_cache_attention_args &a)
{
    const int32_t group = a.n_heads / a.n_kv_heads;
    const int64_t rows = (int64_t)a.max_new * group;
    const auto items_of = [&](int32_t tile_rows) {  // (a product of whole numbers may not fit)
        return (double)a.n_seq * a.n_kv_heads * (double)((rows + tile_rows - 1) / tile_rows);
    };
    // (m_tokens bounds what sequences of different lengths have together: half a tile more each)
    const auto real_of = [&](int32_t tile_rows) {
        return std::min(items_of(tile_rows), (double)a.n_kv_heads * ((double)a.m_tokens * group / tile_rows + 0.5 * a.n_seq));
    };
    // Tiles of 16 rows with the keys split as far as it takes, against 64 or 128 rows that share a chunk of keys (12 heads
    // of 64): 48 queries over 8192 keys (36 tiles of 16 rows) 15 us against 20, 8 times 48 over 2048 (288) 22 against 26,
    // 512 over 8192 (384) 42 against 42, 32 times 128 over 384 (eight times as many) 28 against 17; 8 heads of 128 that 4
    // share, 8 times 64 over 4096 (1024) 101 against 77.
    AttentionPlan p{rows > 16 && items_of(16) > 384, false, false, 16, 1, 0, 0};
    if (p.prompt) {
        // 64 rows, which two waves on either half of the chunks have, against 128 in four waves: half the chunks one after
        // another, where those of the longest sequence are what a call waits for, for twice as many workgroups, of which
        // 768 run at a time (12 heads of 64, tiles of 128; * 16 heads that share 4): 8 times 512 (384 tiles) 15 us against
        // 18, 32 times 128 over 384 (384) 16.8 against 18.2, 16 ragged ones to 2560 keys (429) 36 against 49, 40 times 128
        // over 384 (480) 21.4 against 19.0, 5 times 1024 (480) 26.4 against 28.8, one of 4096 (512*) 63 against 82, 4 times
        // 1536 (576) 40.5 against 40.0, 2 times 3000 (574) 61 against 67, 4 times 1700 (662) 44 against 41, one of 6144
        // (768*) 129 against 135, 4 times 2048 (768) 56 against 51, one of 8192 (1024*) 218 against 203; without causal,
        // where all tiles are as long, 4 times 2000 of 8 heads of 32 (512) 57 against 52. Wider heads have no room for two
        // sets of chunks.
        const double real = real_of(128);
        p.tile_rows = a.head_dim <= 64 && (rows <= 64 || (real <= 768 && a.max_len > (a.causal ? 12 : 24) * (real - 400))) ? 64 : 128;
    }
    // Keys in parts, where there are too few tiles for the CUs and enough keys to pay for joining them (4 us and more): one
    // query over 131072 keys of 8 heads of 128 in 64 parts 58 us, in 32 58, in 128 61, in one 873; 16 queries over 4096 in 4
    // 35, in one 40; 32 over 384 keys of 12 heads (384 tiles) in one 8.9, in 2 12.0. Of 128 rows: 8 times 64 over 4096 keys
    // of 8 heads of 128 that 4 share (128 tiles) in 3 77, in 6 85, in one 114; 64 times 16 over 1024 (512) in one 47, in
    // 2 69.
    const double all = p.prompt ? real_of(p.tile_rows) : items_of(16);
    const int32_t enough = p.prompt ? 384 : 512, least = p.prompt ? 1024 : 512;
    int64_t want = 1;
    if (all < enough) {
        const int64_t items = std::max<int64_t>((int64_t)all, 1);
        want = std::min<int64_t>((enough + items - 1) / items, ((int64_t)a.max_len + least - 1) / least);
        // (tiles that sequences turn out not to have take workspace, and workgroups that join nothing)
        want = (int64_t)std::min((double)want, 2048 / items_of(p.tile_rows));
    }
    if (want > 1) {
        p.split_keys = (int32_t)((((int64_t)a.max_len + want - 1) / want + 255) / 256 * 256);
        p.splits = (int32_t)(((int64_t)a.max_len + p.split_keys - 1) / p.split_keys);
    }
    // Prompts of different lengths: finding a tile's place takes each workgroup 1 to 1.5 us (32 times 128 over 384 keys 18.4
    // against 16.8; one of 2000 tokens with two short ones 32.5 against 31.4), a good order of 16 ragged ones to 512 tokens
    // behind to 2048 35.5 us against 47, of 64 121 against 137, of 4 in two parts 24.7 against 27.6. A workgroup for every
    // CU needs no order.
    //   Steps, whose lengths only the device knows: sequences of one length go on at once (64 times 4096 of 8 heads of 128
    // 99.5 us against 99.1), ragged ones to 4096 take 55 against 65, 128 of them 119 against 127, 32 to 8192 56 against 72;
    // 40 to 3000 of 12 heads of 64, which could be 184 MB, 29.7 against 28.5.
    const bool differ = p.prompt ? a.m_tokens < (int64_t)a.n_seq * a.max_new && all * p.splits > 256
                                 : (double)a.n_seq * a.n_kv_heads * a.max_len * 2 * a.head_dim >= 0x1p28;
    p.by_length = differ && a.n_seq > 1 && a.n_seq <= kMostSorted;
    // Tiles of a sequence that have workgroups of their own. The kernels take those behind them in turns, which they have
    // to for sequences of more tokens than max_new, so one long prompt beside many steps is no reason to refuse a call.
    const int64_t most = kMostItems / ((int64_t)a.n_seq * a.n_kv_heads * p.splits);
    p.fits = most > 0;
    p.tiles = (int32_t)std::min({(rows + p.tile_rows - 1) / p.tile_rows, most, (int64_t)(p.prompt ? kMostGrid / p.splits : kMostItems)});
    return p;
}

struct AppendPlan {
    bool fits, step, vec;                     // (vec: 8 features a thread of queries and keys, else 2)
    int32_t groups;                           // workgroups for a sequence's groups of 16 slots
    int32_t q_columns, k_columns, v_columns;  // a thread each
    int32_t q_parts, k_parts, parts;          // workgroups of queries, of keys, and of all columns
    int32_t per, v_per;                       // columns of one
};

inline AppendPlan plan_of(const sl_cache_append_args &a)
{
    AppendPlan p{};
    p.vec = a.rope_kind == SL_ROPE_NONE || a.rope_dim % 8 == 0;
    const int32_t width = p.vec ? 8 : 2;
    p.q_columns = a.q ? a.n_heads * (a.head_dim / width) : 0;
    p.k_columns = a.n_kv_heads * (a.head_dim / width);
    p.v_columns = a.n_kv_heads * (a.head_dim / 4);
    p.step = a.max_new == 1;
    // (the first may begin anywhere in 16 slots; a launch of fewer goes through them in turns)
    const int64_t groups = p.step ? 1 : std::min<int64_t>(((int64_t)a.max_new + 30) / 16, kMostGrid);
    // Columns of a workgroup: in a step one a thread; else as many as leave 4096 workgroups, since each of them computes
    // its tokens' angles (4 x 4096 tokens of 32 heads of 128 that 4 share: 99.5 us from fp32 and 54 from int8; with 1024
    // 105.8 and 52, with 16384 98 and 73; ragged prompts, which have fewer in all, 17.7 to 17.8).
    const auto even = [](int32_t columns, int32_t most) {  // in equal parts of at most so many
        const int32_t parts = std::max((columns + most - 1) / most, 1);
        return std::max((columns + parts - 1) / parts, 1);
    };
    const double tokens = std::min((double)groups * a.n_seq, (double)a.m_tokens / 16 + a.n_seq);
    int32_t most = 256;
    if (!p.step)
        while (most > 64 && tokens * (p.q_columns + p.k_columns + p.v_columns) / most < 4096) most /= 2;
    p.per = even(std::max(p.q_columns, p.k_columns), most);
    p.v_per = even(p.v_columns, most);
    p.q_parts = (p.q_columns + p.per - 1) / p.per;
    p.k_parts = (p.k_columns + p.per - 1) / p.per;
    p.parts = p.q_parts + p.k_parts + (p.v_columns + p.v_per - 1) / p.v_per;
    // (as cache_attention's tiles: what has no workgroup of its own is done in turns)
    const int64_t room = kMostItems / ((int64_t)a.n_seq * p.parts);
    p.fits = room > 0;
    p.groups = (int32_t)std::min(groups, room);
    return p;
}

}  // namespace sl
