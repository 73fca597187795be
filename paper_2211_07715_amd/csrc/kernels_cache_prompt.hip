// cache_attention for many queries a sequence (gfx950).
//
// The products, the integer scores under the exponential and the two 16-bit parts
// of a weight are those of attention_run (kernels_attention.hip). What differs:
//   queries   a row of the 32-row tiles is a (token, head of the key head's group)
//             pair, so that heads that share keys and values share their chunks;
//   keys      a chunk of 64 is four groups of 16 tokens, each in one page: wave w
//             of a workgroup brings in group w, whose page is then one number for
//             all its lanes. Keys go straight to LDS; the row of LDS that a key
//             takes is chosen so that a lane's scores are of keys whose values lie
//             together, as a page has them: 16 values of a feature are read as 16
//             bytes, turned into 16-bit floats and stored as two pieces, without a
//             transpose;
//   masks     chunks that every query of a wave sees whole go through a loop that
//             masks nothing; the others (the newest tokens' own, a sequence's last,
//             one with a page that is none) and those that move m a step at a time;
//   remainder the second 16 bits of a weight are what the first, cut, leave of it: a
//             mixed multiply-add takes them from the packed first ones (212 us against
//             199.7 for 8192 tokens of 16 heads on 4).
//
// What bounds it: of the 1680 cycles that a SIMD takes for a chunk and a wave of 8192
// tokens (causal, 16 heads of 64 on 4) vector instructions are active in up to 1070
// (counted in steps of 4 cycles) and matrix ones run in 635; three waves a SIMD
// overlap them in part. Half chunks, for four waves a SIMD, took 200 to 211 us against
// 204, and for heads of 128 (three waves against two) 170 to 184 against 187 in a
// prompt of 4096 tokens of 32 heads, but 7 to 12 % more in shorter ones. Two tiles of
// queries a wave 250 against 227 at the time. A prompt of a few chunks is the chain of
// its loads and the first chunk's steps: of 16.7 us for 32 times 128 queries over 384
// keys two thirds are not the chunks'.
//
// Measured, replayed from a graph, causal: 8192 tokens of 16 heads of 64 on 4 193 to
// 228 us on different cards (600 to 710 TOP/s), 4096 of 32 heads of 128 on 8 170 to 199,
// 16 ragged prompts of up to 512 tokens behind up to 2048, 12 heads of 64, 36 (320),
// 32 x 128 queries over 384 keys 16.7 (290). Two chunks between barriers took 203 to 210
// us for 204, and sums of weights by 4x4 matrix instructions 220.
#include <hip/hip_runtime.h>

#include "cache_device.h"

namespace sl {

namespace {

// N: 32-feature tiles of a head. A wave has 32 queries; RW waves share a chunk of
// keys, and the 4 / RW sets of them in a workgroup have the same queries and take
// turns at the chunks, until their m, l and O meet in LDS at the end.
template <int N, int RW>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(N <= 2 ? 3 : 2)))
void cache_prompt_kernel(const CacheArgs a)
{
    constexpr int D = 32 * N, PR = N <= 2 ? 2 * N : 8;  // 16-byte pieces of a key's row in LDS
    constexpr int KS = 16 * PR, VS = 2 * kChunk, KB = kChunk * KS, BUF = KB + D * VS;
    constexpr int KP = (16 * PR + 63) / 64, VP = (D + 63) / 64;  // a lane's pieces of 16 tokens' keys and values
    constexpr int KN = N == 3 ? 4 : N;  // whose swap a key's row takes
    constexpr int KW = 4 / RW, TQ = 32 * RW;
    constexpr int G = 4 / RW;  // groups of 16 tokens of a chunk that a wave brings in
    static_assert(KW * 2 * BUF >= (KW - 1) * RW * 4096 * N, "the parts' O");
    __shared__ __attribute__((aligned(16))) char all_lds[KW * 2 * BUF];
    const int lane = threadIdx.x & 63, half = lane >> 5, n32 = lane & 31;
    const int number = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = number % RW, part = number / RW;
    char *lds = all_lds + part * 2 * BUF;
    // Tiles that see the most keys begin first: every sequence's last one, then the ones before them, or, where sequences
    // differ in length and are few, in that very order (nth_longest). With several sequences every second 256 workgroups
    // go backwards (in eights, so that an XCD keeps its heads): their CUs have work of the 256 before them, and what is
    // long there meets what is short. (16 sequences of up to 512 tokens behind up to 2048, 12 heads: 55 us in the order of
    // sequences, 47 with every second 256 backwards, 35.5 sorted; one of 8192, in order of length as it is: 213 backwards,
    // 204 not.)
    uint32_t head = blockIdx.x, nth = blockIdx.y, turn = blockIdx.z;
    if (gridDim.y > 1) {
        const uint32_t xy = gridDim.x * gridDim.y, number = head + gridDim.x * nth + xy * turn, of = number % 256;
        if ((number / 256 & 1) && number - of + 256 <= xy * gridDim.z) {
            const uint32_t to = number - of + 248 - (of & ~7u) + of % 8, in = to % xy;
            turn = to / xy;
            nth = in / gridDim.x;
            head = in - nth * gridDim.x;
        }
    }
    int32_t seq, from_last, split, b0, b1, len;
    if (a.by_length) {
        const uint32_t rest = nth + gridDim.y * turn;
        const int32_t tile = a.splits == 1 ? rest : rest / (uint32_t)a.splits;
        const Place at = a.n_seq <= 64 ? nth_longest(a, Lengths<1>(a, lane), tile, TQ)
                                       : nth_longest(a, Lengths<kMostSorted / 64>(a, lane), tile, TQ);
        if (at.seq < 0) return;
        seq = at.seq;
        from_last = at.from_last;
        split = rest - tile * a.splits;
        b0 = at.start;
        b1 = at.end;
        len = at.len;
    } else {
        seq = a.seq0 + nth;
        from_last = a.splits == 1 ? turn : turn / (uint32_t)a.splits;
        split = turn - from_last * a.splits;
        b0 = ((ScalarTable)(uintptr_t)a.seq_start)[seq];
        b1 = ((ScalarTable)(uintptr_t)a.seq_start)[seq + 1];
        len = ((ScalarTable)(uintptr_t)a.kv_len)[seq];
    }
    const int32_t kv = head;
    // (without pages nothing is taken from it; the read has to be somewhere)
    const int32_t *row_of_table = a.max_pages ? a.page_table + (int64_t)seq * a.max_pages : a.kv_len;
    const ScalarTable table = (ScalarTable)(uintptr_t)row_of_table;
    const int32_t last_entry = max(a.max_pages - 1, 0);
    // numbers of a chunk's four pages: asked for (all at once, well ahead), and then taken: the wave's own groups', and
    // which of the four are none
    int32_t asked[4], own[G];
    uint32_t none;
    const auto ask = [&](int32_t c) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) asked[j] = table[min((kChunk * c + 16 * j) >> a.shift, last_entry)];
    };
    const auto take = [&]() __attribute__((always_inline)) {
        none = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool there = (uint32_t)asked[j] < (uint32_t)a.n_pages;
            none |= there ? 0u : 1u << j;
            if (j / G == wave) own[j % G] = there ? asked[j] : 0;
        }
    };
    ask(split * (a.split_keys / kChunk) + part);
    // (here they are all waited for, instead of one after the other)
    asm volatile("" : "+s"(asked[0]), "+s"(asked[1]), "+s"(asked[2]), "+s"(asked[3]), "+s"(b0), "+s"(b1), "+s"(len));
    const Tokens tk = tokens_between(b0, b1, a.m);
    len = max(len, 0);
    const int64_t rows = (int64_t)tk.n * a.group;
    const int32_t cached = (int32_t)min((int64_t)len, (int64_t)a.max_pages << a.shift);
    const int64_t head_bytes = (int64_t)a.hd << a.shift, page_bytes = 2 * a.n_kv * head_bytes;
    const int8_t *keys = a.cache + kv * head_bytes, *values = keys + a.n_kv * head_bytes;
    const int32_t in_mask = (1 << a.shift) - 1;

    // A lane's pieces of its wave's 16 tokens: bytes from the first one's, and where they go. Row 8 i + 4 h + b of 16 is
    // key 8 h + 4 i + b, as a lane half h of the scores has them.
    uint32_t koff[KP], vdst[VP];
    bool kmine[KP], vmine[VP];
#pragma unroll
    for (int i = 0; i < KP; ++i) {
        const int p = lane + 64 * i, row = p / PR;  // (every group of 16 rows has the same swaps)
        const int piece = p % PR ^ kswap<KN>(row), key = (row & 3) | (row & 4) << 1 | (row & 8) >> 1;
        kmine[i] = p < 16 * PR && 16 * piece < a.hd;
        koff[i] = (uint32_t)(key * a.hd + 16 * piece);
    }
#pragma unroll
    for (int i = 0; i < VP; ++i) {
        const int d = lane + 64 * i;
        vmine[i] = d < a.hd;
        // (lane half h of the product's rows 8 x + 4 h + b then holds features 16 N h + 16 tile + 4 x + b)
        const int row = 32 * (d / 16 % N) + 8 * (d / 4 % 4) + 4 * (d / (16 * N)) + d % 4;
        vdst[i] = KB + row * VS + 16 * vswap(row);
    }
    i32x4 vreg[G][VP];
    const auto load = [&](int32_t c, char *buf) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int32_t group = wave * G + g;
            const int64_t from = own[g] * page_bytes + ((kChunk * c + 16 * group) & in_mask) * (int64_t)a.hd;
            const auto k = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(keys + from), 0, 0x7fffffff, kRsrcWord3);
            const auto v = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(values + from), 0, 0x7fffffff, kRsrcWord3);
#pragma unroll
            for (int i = 0; i < KP; ++i)
                if (kmine[i]) load_to_lds(k, buf + group * 16 * KS + 1024 * i, koff[i], 0);
#pragma unroll
            for (int i = 0; i < VP; ++i)
                if (vmine[i]) vreg[g][i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(v, 16 * here(lane), 1024 * i, 0));
        }
    };
    const auto stage = [&](char *buf) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                if (!vmine[i]) continue;
                uint32_t out[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // a code c as an unsigned byte c + 128 under the byte 0x64 is the 16-bit float 1152 + c
                    const uint32_t w = (uint32_t)vreg[g][i][j] ^ 0x80808080u, e = 0x64646464u;
                    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
                    out[2 * j] = __builtin_bit_cast(
                        uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(e, w, 0x04010400u)) - bias);
                    out[2 * j + 1] = __builtin_bit_cast(
                        uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(e, w, 0x04030402u)) - bias);
                }
                char *to = buf + (vdst[i] ^ (32 * (wave * G + g))), *to2 = buf + (vdst[i] ^ (32 * (wave * G + g) + 16));
                *reinterpret_cast<i32x4 *>(to) = i32x4{(int)out[0], (int)out[1], (int)out[2], (int)out[3]};
                *reinterpret_cast<i32x4 *>(to2) = i32x4{(int)out[4], (int)out[5], (int)out[6], (int)out[7]};
            }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };

    const int64_t tile0 = (rows + TQ - 1) / TQ - 1 - from_last;
    for (int64_t tile = tile0; tile >= 0; tile -= a.tiles) {
        const int64_t first_row = tile * TQ, end_row = min(first_row + TQ, rows);
        const int32_t i0 = (int32_t)by_group(a, first_row), g0 = (int32_t)(first_row - (int64_t)i0 * a.group);
        // a lane's query: token, or -1, and head
        const auto query = [&](int32_t &head) {
            const int32_t x = wave * 32 + here(n32), y = g0 + x, di = (int32_t)by_group(a, (uint32_t)y);
            head = kv * a.group + (y - di * a.group);
            return first_row + x < end_row ? i0 + di : -1;
        };
        const auto sees = [&](int32_t i) { return a.causal ? min(len - tk.n + i + 1, cached) : cached; };
        const int32_t most = sees((int32_t)by_group(a, end_row - 1));
        // chunks from c0 on: all, or this workgroup's part (one alone has all of a tile that was not said to be there)
        const bool whole = a.splits == 1 || tile >= a.tiles;
        const int32_t c0 = whole ? 0 : split * (a.split_keys / kChunk);
        if (split && (whole || c0 * kChunk >= most)) continue;
        const int32_t all_chunks = (max(most, 0) + kChunk - 1) / kChunk;
        const int32_t n_chunks = whole || split == a.splits - 1 ? all_chunks : min(all_chunks, c0 + a.split_keys / kChunk);
        // keys that the wave's first and last query see
        const int64_t w0 = first_row + wave * 32, w1 = min(w0 + 32, end_row);
        const int32_t least = w0 < end_row ? sees((int32_t)by_group(a, w0)) : 0;
        const int32_t mine =
            w0 < end_row ? min(n_chunks, (max(sees((int32_t)by_group(a, w1 - 1)), 0) + kChunk - 1) / kChunk) : 0;

        int32_t q_head;
        const int32_t mine_i = query(q_head), limit = mine_i >= 0 ? sees(mine_i) : 0x7fffffff;
        i32x4 q[N];
#pragma unroll
        for (int h = 0; h < N; ++h) {
            const int32_t d = 32 * h + 16 * here(half);
            q[h] = i32x4{0, 0, 0, 0};
            if (mine_i >= 0 && d < a.hd)
                q[h] = *reinterpret_cast<const i32x4 *>(a.q + at((int64_t)tk.first + mine_i, q_head * a.hd + d, a.q_cols, a.q_cb));
        }
        f32x16 o[N];
        float l = 0.0f;
        int32_t z = kMagic - kLowest;  // what S starts at: kMagic - m
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
        const auto scores = [&](const char *buf, const i32x16 &from, i32x16 (&s)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                s[kt] = from;
#pragma unroll
                for (int h = 0; h < N; ++h) {
                    const int row = 32 * kt + n32;
                    const i32x4 k = *reinterpret_cast<const i32x4 *>(buf + row * KS + 16 * ((2 * h + half) ^ kswap<KN>(n32)));
                    s[kt] = __builtin_amdgcn_mfma_i32_32x32x32_i8(k, q[h], s[kt], 0, 0, 0);
                }
            }
        };
        const auto from_z = [&]() {
            i32x16 v;
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = z;
            asm volatile("" : "+v"(v));  // 16 registers for the loop over chunks, not 32 moves in it
            return v;
        };
        // keys that the query does not see: minus infinity, as the bits that the scores are
        const auto mask = [&](int32_t c, uint32_t gone, i32x16 (&s)[2]) __attribute__((always_inline)) {
            const int32_t left = limit - kChunk * c - 8 * half;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * kt + 16 * (i / 8) + i % 8 >= left || (gone >> (2 * kt + i / 8) & 1)) s[kt][i] = (int32_t)0xff800000;
        };
        const auto largest = [&](const i32x16 (&s)[2]) __attribute__((always_inline)) {
            int32_t top = 0;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = max(top, s[kt][i]);
            return top;
        };
        const auto raise = [&](int32_t top) __attribute__((always_inline)) {
            const int32_t by = max(pair_max(top) - kMagic, 0);
            const float f = __builtin_amdgcn_exp2f(-(float)by * a.c2);
            z -= by;
            l *= f;
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
            return by;
        };
        f16x8 p[4], p2[4];
        const auto weights = [&](const i32x16 (&s)[2]) __attribute__((always_inline)) {
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {  // 16 keys
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    float e[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int i = 8 * (w & 1) + j + r;
                        e[r] = __builtin_amdgcn_exp2f(fmaf(__int_as_float(s[w / 2][i]), a.c2, a.k2));
                        sum[2 * (w & 1) + r] += e[r];
                    }
                    const f16x2 h = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(e[0], e[1]));
                    float rest[2];
                    asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel_hi:[1,0,0]" : "=v"(rest[0]) : "v"(h), "v"(e[0]));
                    asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(rest[1]) : "v"(h), "v"(e[1]));
                    const f16x2 l2 = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(rest[0], rest[1]));
                    p[w][j] = h[0];
                    p[w][j + 1] = h[1];
                    p2[w][j] = l2[0];
                    p2[w][j + 1] = l2[1];
                }
            }
            return (sum[0] + sum[1]) + (sum[2] + sum[3]);
        };
        const auto multiply = [&](const char *buf) __attribute__((always_inline)) {
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int d = 0; d < N; ++d) {
                    const f16x8 v = *reinterpret_cast<const f16x8 *>(
                        buf + KB + (32 * d + n32) * VS + 16 * ((2 * w + half) ^ vswap(n32)));
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[w], o[d], 0, 0, 0);
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p2[w], o[d], 0, 0, 0);
                }
        };

        int32_t c = c0 + part, buf = 0;
        uint32_t gone = 0;  // which of the chunk's pages are none
        if (c < n_chunks) {
            if (tile != tile0) ask(c);
            take();
            gone = none;
            load(c, lds);
            ask(c + KW);
            stage(lds);
            take();
        }
        __syncthreads();
        // every chunk: the next one's loads, this one's work, then the next one goes to LDS
        const auto bring = [&]() __attribute__((always_inline)) {
            if (c + KW < n_chunks) {
                load(c + KW, lds + (buf ^ BUF));
                ask(c + 2 * KW);
            }
        };
        const auto advance = [&]() __attribute__((always_inline)) {
            buf ^= BUF;
            c += KW;
            gone = none;
            if (c < n_chunks) {
                stage(lds + buf);
                take();
            }
            __syncthreads();
        };
        i32x16 sc[2];
        while (c < mine) {
            bring();
            scores(lds + buf, from_z(), sc);
            // (where the two sides take turns the first chunk is a large part of all, and mostly seen whole; elsewhere the
            // branch costs more than it saves: 32 x 512 tokens of 12 heads 36.8 us against 34.7)
            if (RW == 4 || kChunk * (c + 1) > least || gone) mask(c, gone, sc);
            const int32_t by = raise(largest(sc));
            // (what is masked stays far below everything, as a finite number)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[kt][i] -= by;
            l += weights(sc);
            multiply(lds + buf);
            advance();
            const i32x16 from = from_z();
            while (kChunk * (c + 1) <= least && c < mine && !gone) {
                bring();
                scores(lds + buf, from, sc);
                const float sum = weights(sc);
                if (__any(!(sum < kMostSum))) break;  // (no weight is over 65504 while their sum is below that)
                l += sum;
                // (matrix instructions of one wave before vector ones of another: 4096 tokens of 32 heads of 128 on 8 199 us
                // against 210, 8192 of 16 of 64 on 4 227 against 232)
                __builtin_amdgcn_s_setprio(1);
                multiply(lds + buf);
                __builtin_amdgcn_s_setprio(0);
                advance();
            }
        }
        while (c - part < n_chunks) {  // others' chunks
            bring();
            advance();
        }
        // a lane half holds features 16 N half .. 16 N half + 16 N - 1 of its query
        float sum = pair_sum(l);
        if constexpr (KW > 1) {
            // what the other parts have goes to the first, which puts all on the largest m
            __shared__ int32_t zs[KW - 1][TQ];
            __shared__ float ls[KW - 1][TQ];
            const int row = wave * 32 + n32;
            float *to = reinterpret_cast<float *>(all_lds) + lane;
            if (part) {
                if (half == 0) {
                    zs[part - 1][row] = z;
                    ls[part - 1][row] = sum;
                }
#pragma unroll
                for (int d = 0; d < N; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) to[((part - 1) * RW + wave) * (1024 * N) + 64 * (16 * d + e)] = o[d][e];
            }
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int k = 0; k < KW - 1; ++k) {
                    const int32_t z2 = zs[k][row], least_z = min(z, z2);
                    const float f = __builtin_amdgcn_exp2f(-(float)(z - least_z) * a.c2);
                    const float f2 = __builtin_amdgcn_exp2f(-(float)(z2 - least_z) * a.c2);
                    z = least_z;
                    sum = sum * f + ls[k][row] * f2;
#pragma unroll
                    for (int d = 0; d < N; ++d)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            o[d][e] = o[d][e] * f + to[(k * RW + wave) * (1024 * N) + 64 * (16 * d + e)] * f2;
                }
            }
            if (tile >= a.tiles) __syncthreads();  // (before the next tile's keys come)
            if (part) continue;
        }
        const int32_t i = query(q_head);
        const int h2 = here(half);
        if (!whole) {
            const int row = wave * 32 + here(n32);
            float *rec = a.work + ((((int64_t)seq * a.n_kv + kv) * a.tiles + tile) * a.splits + split) * record(a.hd, TQ);
            if (i < 0) continue;
            if (h2 == 0) {
                reinterpret_cast<int32_t *>(rec)[row] = kMagic - z;
                rec[TQ + row] = sum;
            }
#pragma unroll
            for (int d = 0; d < N; ++d) {
                const int32_t f0 = 16 * N * h2 + 16 * d;
                if (f0 >= a.hd) continue;
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *reinterpret_cast<f32x4 *>(rec + 2 * TQ + (int64_t)row * a.hd + f0 + e) =
                        f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
            }
            continue;
        }
        const float mean = sum > 0.0f ? a.vs / sum : 0.0f, f = mean * a.unit;
        const int32_t cols = a.n_heads * a.hd;
        if (i < 0) continue;
        const int64_t tok = (int64_t)tk.first + i;
#pragma unroll
        for (int d = 0; d < N; ++d) {
            const int32_t f0 = 16 * N * h2 + 16 * d;
            if (f0 >= a.hd) continue;
            if (a.y_f32) {
                float *y = static_cast<float *>(a.y) + tok * cols + q_head * a.hd + f0;
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    *reinterpret_cast<f32x4 *>(y + e) = f32x4{o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]} * mean * a.unit;
            } else {
                i32x4 w;
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    w[e / 4] = (int)pack_bytes(requant_bits(o[d][e], f), requant_bits(o[d][e + 1], f),
                                               requant_bits(o[d][e + 2], f), requant_bits(o[d][e + 3], f));
                *reinterpret_cast<i32x4 *>(static_cast<int8_t *>(a.y) + at(tok, q_head * a.hd + f0, cols, a.y_cb)) = w;
            }
        }
    }
}

template <int N>
void launch_shape(const CacheArgs &a, dim3 grid, hipStream_t s)
{
    if constexpr (N <= 2) {
        if (a.tile_rows == 64) {
            hipLaunchKernelGGL((cache_prompt_kernel<N, 2>), grid, dim3(256), 0, s, a);
            return;
        }
    }
    hipLaunchKernelGGL((cache_prompt_kernel<N, 4>), grid, dim3(256), 0, s, a);
}

}  // namespace

sl_status launch_cache_prompt(const CacheArgs &a, dim3 grid, hipStream_t s)
{
    switch ((a.hd + 31) / 32) {
    case 1: launch_shape<1>(a, grid, s); break;
    case 2: launch_shape<2>(a, grid, s); break;
    case 3: launch_shape<3>(a, grid, s); break;
    default: launch_shape<4>(a, grid, s); break;
    }
    HIP_TRY(hipGetLastError());
    return SL_OK;
}

}  // namespace sl
