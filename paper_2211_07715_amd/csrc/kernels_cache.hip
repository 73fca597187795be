// A decoder's cache (gfx950): cache_append, and cache_attention for few queries a
// sequence. (kernels_cache_prompt.hip has it for many.)
//
// cache_append. Memory bounds it: an element is read once (4 bytes or 1), turned by
// 4 operations and written as one byte. A token's angles serve all its heads, so a
// workgroup computes them once in LDS (position times frequency in 64 bits, reduced
// to quarter turns) and goes through its columns. 16 slots go together, because a
// page holds 16 tokens' codes of a value's feature in 16 bytes; with one token a
// sequence these are single bytes, 16 apart. What a wave's lanes have in common, its
// token, and what its tokens have in common, a lane's features, make up an address,
// so that neither loads nor stores compute one.
//   Measured, replayed from a graph: 4 x 4096 tokens of 32 heads of 128 that 4 share,
// fp32, 97 us (5.18 TB/s; a copy of 1 GiB reaches 5.20), from int8 codes 51 (3.9
// TB/s; vector instructions: 8 an element); 24 ragged prompts of up to 384 tokens of
// 12 heads of 64, int8, 14.4 us; 64 sequences of one token, fp32, 4.3 us, one 3.1 us.
//
// cache_attention, few queries: each key and value byte is read once, for 4
// operations and query head that shares it, so memory bounds it. Nothing passes
// through LDS on the way to the matrix instructions: keys and values lie in a page
// as lanes take them (16 bytes are 16 features of a key, or 16 tokens of a feature).
//   S = K Q^T     int8 x int8 -> int32 on v_mfma_i32_16x16x64_i8, exact
//   P = 2^(c (S - m)), m the largest of a span of 64 keys: as whole numbers of 23
//       bits in three signed bytes
//   O += V^T P^T  int8 x int8 -> int32, exact, a product for each byte
// Values need no conversion, sums of a span are whole numbers, and a span's results
// join the others' in fp32 by their m. Row x of a score tile is the key that makes a
// lane's scores those of the 16 tokens whose values it takes, so weights stay in
// their lane. A column is a (query, head) pair: heads that share keys share the rows.
//   A wave takes every 4th span of 64 keys. Three waves a SIMD, whose loads are all
// under way before a span's first product, keep memory busy: asking for the next
// span during the products of one took registers for two waves and gave the same
// rate; spans of 128 keys gave the same (99.6 us) and cost short sequences (5.4
// against 4.7 us).
//   Measured, replayed from a graph: 64 x 4096 tokens of 8 key heads of 128 with 4
// query heads each 98.5 us (5.45 TB/s; reading alone reaches 6.4), 64 x 16384 374 (5.7),
// 131072 tokens 57 to 61 (50 and 5 for the two launches), 24 ragged sequences of up
// to 3001 tokens of 8 heads of 96 18.7 (2.75 TB/s: 16 and 4), 64 ragged ones of
// up to 4096 of 8 heads of 128 55 (4.6), 32 x 384 tokens of 12 heads of 64 8.4, 128
// tokens 4.7. Vector instructions are active 30 % of the time
// in the first, matrix ones 7 %.
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <charconv>
#include <type_traits>

#include "cache_device.h"
#include "cache_plan.h"
#include "encoder.h"

namespace sl {

namespace {

// --- cache_append --------------------------------------------------------------

struct AppendArgs {
    const int8_t *x;
    int8_t *q, *cache;
    const int32_t *seq_start, *kv_len, *page_table, *positions;
    const float *inv_freq;
    int64_t m;
    int32_t seq0, max_pages, n_pages, shift;  // 1 << shift: tokens of a page
    int32_t nh, nkv, hd, x_cb, q_cb;
    int32_t x_step, q_step;                   // bytes of a token's row, or of 16 tokens' blocks
    uint32_t values;                          // bytes from a page's keys to its values
    int64_t page_bytes;
    int32_t half, split;                      // rotated pairs of a head; 1: (j, j + half), 0: (2 j, 2 j + 1)
    int32_t q_columns, k_columns, v_columns;  // a thread each
    int32_t q_parts, k_parts, per, v_per;     // workgroups of queries and of keys, and columns of one
    float rope_factor, fq, fk, fv;            // f*: from x's unit to the codes'
    float inv_qk, inv_value, inv_half;        // 1 / columns of a head, and of its rotated pairs
};

__device__ __forceinline__ f32x4 codes_to_float(uint32_t w)
{
    return f32x4{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
}

// Codes of 4 values. 1.5 * 2^23 more than value * f is rounded to a whole number, whose
// low byte is the code once it is within 127 of that.
__device__ __forceinline__ uint32_t code_bits(float v, float f)
{
    return __float_as_uint(__builtin_amdgcn_fmed3f(fmaf(v, f, kMagicF), kMagicF - 127.0f, kMagicF + 127.0f));
}
__device__ __forceinline__ uint32_t codes_of(f32x4 v, float f)
{
    return pack_bytes(code_bits(v[0], f), code_bits(v[1], f), code_bits(v[2], f), code_bits(v[3], f));
}

// 4 x 4 bytes: byte j of word e becomes byte e of word j.
__device__ __forceinline__ void transpose_bytes(uint32_t (&w)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// The rows of some tokens, the same for a wave: the first one's, and where others begin from there. (64 bits for one of
// them only: addresses of four rows took 200 scalar instructions a wave.)
struct Rows {
    int8_t *base;
    int32_t step, phase;  // phase: the first one's place in its block of 16 tokens, or -1 for whole rows
    __device__ __forceinline__ Rows(const int8_t *x, int32_t t, int32_t cb, int32_t bytes)
        : base(const_cast<int8_t *>(x) + (int64_t)(cb ? t >> 4 : t) * bytes), step(bytes), phase(cb ? t & 15 : -1)
    {
    }
    __device__ __forceinline__ int8_t *at(int32_t j) const
    {
        const int32_t i = phase + j;
        return base + (phase < 0 ? j * step : (i >> 4) * step + (i & 15) * 32);
    }
};
// A feature's place from its token's first.
__device__ __forceinline__ uint32_t feature_offset(int32_t c, int32_t cb, int32_t size)
{
    return cb ? (uint32_t)(c >> 5) * 512 + (c & 31) : (uint32_t)c * size;
}

// number / by and what is left of it; number is under 2^23 and its quotient in fp32 off by less than one.
__device__ __forceinline__ void divide(int32_t number, int32_t by, float inv, int32_t &quotient, int32_t &rest)
{
    quotient = (int32_t)(((float)number + 0.5f) * inv);
    rest = number - quotient * by;
    const int32_t more = rest < 0 ? -1 : rest >= by ? 1 : 0;
    quotient += more;
    rest -= more * by;
}

// What a thread does: a column, which is 8 features of a query or key head (VEC:
// rope_dim is a multiple of 8, so that 4 features of both halves of pairs lie
// together; else 2 features), or 4 features of a value head. A workgroup's columns
// are all of queries, of keys or of values.
template <bool F32, bool VEC>
struct PairColumn {
    static constexpr int U = VEC ? 8 : 2;
    using Raw = std::conditional_t<VEC, std::conditional_t<F32, f32x4, uint32_t>, std::conditional_t<F32, float, int8_t>>;
    int32_t w0;               // first angle
    bool turned;
    uint32_t x0, x1, d0, d1;  // bytes of both parts from a token's first: in x, and where their codes go
    __device__ __forceinline__ PairColumn(const AppendArgs &p, int32_t number, bool keys)
    {
        int32_t head, k;
        divide(number, p.hd / U, p.inv_qk, head, k);
        w0 = VEC ? 4 * k : k;
        turned = w0 < p.half;
        const bool apart = turned && p.split;
        const int32_t c0 = apart ? w0 : U * k, c1 = apart ? w0 + p.half : c0 + U / 2;
        const int32_t x_head = (keys ? p.nh + head : head) * p.hd;
        x0 = feature_offset(x_head + c0, p.x_cb, F32 ? 4 : 1);
        x1 = feature_offset(x_head + c1, p.x_cb, F32 ? 4 : 1);
        d0 = keys ? (uint32_t)(head << p.shift) * p.hd + c0 : feature_offset(head * p.hd + c0, p.q_cb, 1);
        d1 = keys ? d0 + (c1 - c0) : feature_offset(head * p.hd + c1, p.q_cb, 1);
    }
    __device__ __forceinline__ static Raw load(const int8_t *row, uint32_t by) { return *reinterpret_cast<const Raw *>(row + by); }
    // a token's codes: cs, sn are its angles' cosines and sines, its row of codes begins at `to`
    __device__ __forceinline__ void put(const AppendArgs &p, Raw r0, Raw r1, const float *cs, const float *sn, int8_t *to,
                                        float f) const
    {
        if constexpr (VEC) {
            f32x4 y0, y1;
            if constexpr (F32) {
                y0 = r0;
                y1 = r1;
            } else {
                y0 = codes_to_float(r0);
                y1 = codes_to_float(r1);
            }
            if (turned) {
                const f32x4 c = *reinterpret_cast<const f32x4 *>(cs + w0), s = *reinterpret_cast<const f32x4 *>(sn + w0);
                const f32x4 x = y0, y = y1;
                if (p.split) {
                    y0 = x * c - y * s;
                    y1 = y * c + x * s;
                } else {
                    y0 = f32x4{x[0] * c[0] - x[1] * s[0], x[1] * c[0] + x[0] * s[0], x[2] * c[1] - x[3] * s[1],
                               x[3] * c[1] + x[2] * s[1]};
                    y1 = f32x4{y[0] * c[2] - y[1] * s[2], y[1] * c[2] + y[0] * s[2], y[2] * c[3] - y[3] * s[3],
                               y[3] * c[3] + y[2] * s[3]};
                }
            }
            *reinterpret_cast<uint32_t *>(to + d0) = codes_of(y0, f);
            *reinterpret_cast<uint32_t *>(to + d1) = codes_of(y1, f);
        } else {
            float x = (float)r0, y = (float)r1;
            if (turned) {
                const float c = cs[w0], s = sn[w0], x2 = x * c - y * s;
                y = y * c + x * s;
                x = x2;
            }
            to[d0] = (int8_t)code_bits(x, f);
            to[d1] = (int8_t)code_bits(y, f);
        }
    }
};

template <bool F32>
struct ValueColumn {
    using Raw = std::conditional_t<F32, f32x4, uint32_t>;
    uint32_t x0, d0;  // bytes from a token's first in x, and from a page's first value in a group of 16 tokens
    __device__ __forceinline__ ValueColumn(const AppendArgs &p, int32_t number)
    {
        int32_t head, c;
        divide(number, p.hd / 4, p.inv_value, head, c);
        c *= 4;
        x0 = feature_offset((p.nh + p.nkv + head) * p.hd + c, p.x_cb, F32 ? 4 : 1);
        d0 = (uint32_t)(head << p.shift) * p.hd + c * 16;
    }
    __device__ __forceinline__ Raw load(const int8_t *row) const { return *reinterpret_cast<const Raw *>(row + x0); }
    __device__ __forceinline__ static uint32_t codes(const AppendArgs &p, Raw r)
    {
        if constexpr (F32)
            return codes_of(r, p.fv);
        else
            return codes_of(codes_to_float(r), p.fv);
    }
};

// rope_factor times the cosine and sine of pos * inv_freq[w]. The angle is reduced to
// quarter turns in 64 bits; within an eighth of a turn, |x| <= pi / 4, the Taylor sums
// to x^9 and x^10 are within 2^-29 and 2^-31.
__device__ __forceinline__ void angle(const AppendArgs &p, double pos, int32_t w, float &c, float &s)
{
    const double quarters = pos * (double)p.inv_freq[w] * 0.63661977236758134308, whole = rint(quarters);
    const float x = (float)(quarters - whole) * 1.57079632679489662f, x2 = x * x;
    const uint32_t turn = (uint32_t)(int64_t)whole;
    float sine = fmaf(x2, 1.0f / 362880.0f, -1.0f / 5040.0f);
    sine = fmaf(x2, sine, 1.0f / 120.0f);
    sine = fmaf(x2, sine, -1.0f / 6.0f);
    sine = fmaf(x * x2, sine, x);
    float cosine = fmaf(x2, -1.0f / 3628800.0f, 1.0f / 40320.0f);
    cosine = fmaf(x2, cosine, -1.0f / 720.0f);
    cosine = fmaf(x2, cosine, 1.0f / 24.0f);
    cosine = fmaf(x2, cosine, -0.5f);
    cosine = fmaf(x2, cosine, 1.0f);
    c = p.rope_factor * (turn & 1 ? sine : cosine) * ((turn + 1) & 2 ? -1.0f : 1.0f);
    s = p.rope_factor * (turn & 1 ? cosine : sine) * (turn & 2 ? -1.0f : 1.0f);
}

// The lengths of a sequence: its tokens of the call and its cached ones.
__device__ __forceinline__ Tokens lengths(const AppendArgs &p, int32_t seq, int32_t &len)
{
    int32_t b0 = ((ScalarTable)(uintptr_t)p.seq_start)[seq], b1 = ((ScalarTable)(uintptr_t)p.seq_start)[seq + 1];
    len = ((ScalarTable)(uintptr_t)p.kv_len)[seq];
    asm volatile("" : "+s"(b0), "+s"(b1), "+s"(len));  // (here they are all waited for, instead of one after the other)
    len = max(len, 0);
    return tokens_between(b0, b1, p.m);
}

// The page that holds a slot, or NULL.
__device__ __forceinline__ int8_t *page_of(const AppendArgs &p, int32_t seq, int32_t slot)
{
    const int32_t entry = slot >> p.shift;
    if (slot < 0 || entry >= p.max_pages) return nullptr;
    const int32_t number = ((ScalarTable)(uintptr_t)p.page_table)[(int64_t)seq * p.max_pages + entry];
    if ((uint32_t)number >= (uint32_t)p.n_pages) return nullptr;
    return p.cache + number * p.page_bytes;
}

// Which columns a workgroup has: `first` to `end` of the queries (0), keys (1) or values (2).
struct Share {
    int32_t kind, first, end;
};
__device__ __forceinline__ Share share_of(const AppendArgs &p, int32_t part)
{
    if (part < p.q_parts) return {0, part * p.per, min((part + 1) * p.per, p.q_columns)};
    part -= p.q_parts;
    if (part < p.k_parts) return {1, part * p.per, min((part + 1) * p.per, p.k_columns)};
    part -= p.k_parts;
    return {2, part * p.v_per, min((part + 1) * p.v_per, p.v_columns)};
}

// One token a sequence: a thread a column, its loads under way while the angles are computed.
template <bool F32, bool VEC>
__global__ __launch_bounds__(256) void cache_append_step_kernel(const AppendArgs p)
{
    __shared__ __attribute__((aligned(16))) float cs[64], sn[64];
    const int tid = threadIdx.x, seq = p.seq0 + blockIdx.z;
    const Share my = share_of(p, blockIdx.x);
    const int32_t column = my.first + tid;
    const bool mine = column < my.end;
    int32_t len;
    const Tokens tk = lengths(p, seq, len);
    for (int32_t i = 0; i < tk.n; ++i) {  // (one, unless a sequence has more than was said)
        const int32_t t = tk.first + i, slot = len - tk.n + i;
        const int8_t *row = Rows(p.x, t, p.x_cb, p.x_step).at(0);
        const int32_t in_page = slot & ((1 << p.shift) - 1);
        if (my.kind == 2) {
            const ValueColumn<F32> col(p, column);
            typename ValueColumn<F32>::Raw r{};
            if (mine) r = col.load(row);
            int8_t *page = page_of(p, seq, slot);
            if (!page || !mine) continue;
            int8_t *to = page + p.values + (in_page & ~15) * p.hd + (in_page & 15);
            const uint32_t w = col.codes(p, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) (to + 16 * e)[col.d0] = (int8_t)(w >> (8 * e));
        } else {
            const PairColumn<F32, VEC> col(p, column, my.kind == 1);
            typename PairColumn<F32, VEC>::Raw r0{}, r1{};
            if (mine) {
                r0 = col.load(row, col.x0);
                r1 = col.load(row, col.x1);
            }
            int8_t *page = my.kind ? page_of(p, seq, slot) : nullptr;
            if (p.half) {
                __syncthreads();
                if (tid < p.half) angle(p, p.positions ? (double)p.positions[t] : (double)slot, tid, cs[tid], sn[tid]);
                __syncthreads();
            }
            if (!mine || (my.kind && !page)) continue;
            col.put(p, r0, r1, cs, sn, my.kind ? page + in_page * p.hd : Rows(p.q, t, p.q_cb, p.q_step).at(0),
                    my.kind ? p.fk : p.fq);
        }
    }
}

// Many tokens a sequence. One workgroup: the tokens in 16 consecutive slots, which is
// what lies together in the values' pages, and some columns, 64 at a time; a wave has
// 4 of the slots, whose loads are all under way before any is used.
template <bool F32, bool VEC>
__global__ __launch_bounds__(256) void cache_append_kernel(const AppendArgs p)
{
    __shared__ __attribute__((aligned(16))) float cs[16][64], sn[16][64];
    __shared__ __attribute__((aligned(16))) uint32_t words[4][64][4];  // 4 tokens' codes of a value's feature
    const int tid = threadIdx.x, lane = tid & 63, quad = __builtin_amdgcn_readfirstlane(tid >> 6), seq = p.seq0 + blockIdx.z;
    const Share my = share_of(p, blockIdx.x);
    int32_t len;
    const Tokens tk = lengths(p, seq, len);
    const int32_t p0 = len - tk.n, ahead = p0 & 15;  // the first token's slot, and the slots before it in its 16
    const int32_t groups = tk.n ? (tk.n + ahead + 15) >> 4 : 0;
    for (int32_t g = blockIdx.y; g < groups; g += gridDim.y) {
        // slots from .. to - 1 of the 16 have a token, j0 .. j1 - 1 of the wave's 4
        const int32_t s0 = p0 - ahead + 16 * g, from = g ? 0 : ahead, to = min(tk.n + ahead - 16 * g, 16);
        const int32_t j0 = min(max(from - 4 * quad, 0), 4), j1 = min(max(to - 4 * quad, 0), 4);
        const int32_t t0 = tk.first - ahead + 16 * g + 4 * quad;  // the token of the wave's first slot
        const Rows x(p.x, t0, p.x_cb, p.x_step);
        const int32_t in_page = s0 & ((1 << p.shift) - 1);
        int8_t *page = my.kind ? page_of(p, seq, s0) : nullptr;
        if (my.kind == 2) {
            if (!page) continue;
            int8_t *group = page + p.values + in_page * p.hd;
            for (int32_t column = my.first; column < my.end; column += 64) {
                const bool mine = column + lane < my.end;
                const ValueColumn<F32> col(p, column + lane);
                typename ValueColumn<F32>::Raw r[4]{};
                if (j1 - j0 == 4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (mine) r[j] = col.load(x.at(j));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (mine && j >= j0 && j < j1) r[j] = col.load(x.at(j));
                }
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = col.codes(p, r[j]);
                // features e = 0 .. 3, a word of 4 tokens each
                transpose_bytes(w);
                if (to - from == 16) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) words[e][lane][quad] = w[e];
                    __syncthreads();
                    if (mine)
                        *reinterpret_cast<i32x4 *>(group + 16 * quad + col.d0) =
                            *reinterpret_cast<const i32x4 *>(words[quad][lane]);
                    __syncthreads();
                } else if (mine) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        int8_t *at = group + 16 * e + 4 * quad + col.d0;
                        if (j1 - j0 == 4)
                            *reinterpret_cast<uint32_t *>(at) = w[e];
                        else
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (j >= j0 && j < j1) at[j] = (int8_t)(w[e] >> (8 * j));
                    }
                }
            }
            continue;
        }
        if (my.kind && !page) continue;
        if (p.half) {
            __syncthreads();
            // (a wave the angles of its own slots; their number divides by no more than 64 rotated pairs)
            for (int32_t i = lane; i < 4 * p.half; i += 64) {
                const int32_t j = (int32_t)(((float)i + 0.5f) * p.inv_half), w = i - j * p.half;
                if (j >= j0 && j < j1)
                    angle(p, (double)(p.positions ? p.positions[t0 + j] : s0 + 4 * quad + j), w,
                          cs[4 * quad + j][w], sn[4 * quad + j][w]);
            }
            __syncthreads();
        }
        const Rows y = my.kind ? Rows(page, in_page + 4 * quad, 0, p.hd) : Rows(p.q, t0, p.q_cb, p.q_step);
        const float f = my.kind ? p.fk : p.fq;
        for (int32_t column = my.first + lane; column < my.end; column += 64) {
            const PairColumn<F32, VEC> col(p, column, my.kind == 1);
            if (j1 - j0 == 4) {
                typename PairColumn<F32, VEC>::Raw r0[4], r1[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    r0[j] = col.load(x.at(j), col.x0);
                    r1[j] = col.load(x.at(j), col.x1);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) col.put(p, r0[j], r1[j], cs[4 * quad + j], sn[4 * quad + j], y.at(j), f);
            } else {
                typename PairColumn<F32, VEC>::Raw r0[4]{}, r1[4]{};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j < j0 || j >= j1) continue;
                    r0[j] = col.load(x.at(j), col.x0);
                    r1[j] = col.load(x.at(j), col.x1);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j >= j0 && j < j1) col.put(p, r0[j], r1[j], cs[4 * quad + j], sn[4 * quad + j], y.at(j), f);
            }
        }
    }
}

// --- cache_attention, few queries a sequence ---------------------------------------

constexpr int kWaves = 4;  // of a workgroup, which share its keys
constexpr int kSpan = 64;  // keys that a wave takes at a time

__device__ __forceinline__ int quad_max(int v)  // over lanes 16 and 32 apart
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((int)a[0], (int)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((int)b[0], (int)b[1]);
}
__device__ __forceinline__ float quad_sum(float v)
{
    int i = __float_as_int(v);
    const auto a = __builtin_amdgcn_permlane16_swap(i, i, false, false);
    i = __float_as_int(__int_as_float(a[0]) + __int_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    return __int_as_float(b[0]) + __int_as_float(b[1]);
}

// A weight of 0 .. 1 times kLargest plus kDigits is a float whose mantissa is the weight's whole number + 0x8080: its low
// three bytes are three digits to the base 256, the lower two of them 128 too large.
constexpr float kDigits = 8388608.0f + 32896.0f;
constexpr uint32_t kDigitsBits = 0x4B008080u;
constexpr float kLargest = 8355000.0f;  // (and 2^23 - 0x8080 more than it, by enough for an exponential over 1)
constexpr int32_t kNone = -(1 << 30);  // m without a key

// One output row's share: query row, 4 features from c on
__device__ __forceinline__ void store_row(const CacheArgs &a, int64_t tok, int32_t head, int32_t c, f32x4 v, float l)
{
    const float g = l > 0.0f ? a.vs / l : 0.0f;  // (under 4, as unit times it is finite)
    const int32_t cols = a.n_heads * a.hd;
    if (a.y_f32)
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + tok * cols + head * a.hd + c) = v * g * a.unit;
    else
        *reinterpret_cast<uint32_t *>(static_cast<int8_t *>(a.y) + at(tok, head * a.hd + c, cols, a.y_cb)) =
            codes_of(v, g * a.unit);
}

// SORTED: where sequences turn out to differ in length, those that see the most keys come first.
template <int F, bool SORTED>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(3))) void cache_split_kernel(const CacheArgs a)
{
    constexpr int N = (F + 3) / 4, HD = 16 * F, FB = 2;
    __shared__ __attribute__((aligned(16))) float parts[kWaves][F * 4][64];
    __shared__ int32_t ms[kWaves][16];
    __shared__ float ls[kWaves][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, h = lane >> 4;
    int32_t split = blockIdx.z, seq = a.seq0 + blockIdx.y;
    int32_t kv = a.tiles == 1 ? blockIdx.x : blockIdx.x / (uint32_t)a.tiles, tile0 = blockIdx.x - kv * a.tiles;
    const int32_t last_entry = a.max_pages - 1, in_mask = (1 << a.shift) - 1;
    // pages of the 16 keys that the lane's row of the scores' left operand and its values come from
    int32_t pk = -1, pv = -1;
    const auto entries = [&](int32_t kb) __attribute__((always_inline)) {
        const int32_t *table = a.page_table + (int64_t)seq * a.max_pages;
        pk = table[min((kb + 16 * (r >> 2)) >> a.shift, last_entry)];
        pv = table[min((kb + 16 * h) >> a.shift, last_entry)];
    };
    if (a.max_pages) entries(split * a.split_keys + wave * kSpan);  // (on their way with the lengths)
    int32_t b0, b1, len;
    if constexpr (!SORTED) {
        b0 = ((ScalarTable)(uintptr_t)a.seq_start)[seq];
        b1 = ((ScalarTable)(uintptr_t)a.seq_start)[seq + 1];
        len = ((ScalarTable)(uintptr_t)a.kv_len)[seq];
        asm volatile("" : "+s"(b0), "+s"(b1), "+s"(len));  // (here they are all waited for, instead of one after the other)
    } else {
        const auto place = [&](const auto &all, auto sets) __attribute__((always_inline)) {
            if (all.equal(a, lane)) {
#pragma unroll
                for (int g = 0; g < sets; ++g) {
                    if (seq / 64 != g) continue;
                    b0 = __builtin_amdgcn_readlane(all.start[g], seq % 64);
                    b1 = __builtin_amdgcn_readlane(all.end[g], seq % 64);
                    len = __builtin_amdgcn_readlane(all.len[g], seq % 64);
                }
                return true;
            }
            // (every second 256 workgroups backwards, as prompts have them)
            uint32_t number = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
            const uint32_t of = number % 256;
            if ((number / 256 & 1) && number - of + 256 <= gridDim.x * gridDim.y * gridDim.z)
                number = number - of + 248 - (of & ~7u) + of % 8;
            const uint32_t rest = number / (uint32_t)a.n_kv, most = gridDim.y * a.tiles;
            kv = number - rest * a.n_kv;
            split = a.splits == 1 ? 0 : rest / most;
            const Place at = nth_longest(a, all, rest - split * most, 16);
            if (at.seq < 0) return false;
            seq = at.seq;
            b0 = at.start;
            b1 = at.end;
            len = at.len;
            tile0 = (int32_t)((((int64_t)tokens_between(b0, b1, a.m).n * a.group + 15) / 16 - 1 - at.from_last) % a.tiles);
            if (a.max_pages) entries(split * a.split_keys + wave * kSpan);
            return true;
        };
        if (a.n_seq <= 64) {
            if (!place(Lengths<1>(a, lane), std::integral_constant<int, 1>{})) return;
        } else {
            if (!place(Lengths<kMostSorted / 64>(a, lane), std::integral_constant<int, kMostSorted / 64>{})) return;
        }
    }
    const Tokens tk = tokens_between(b0, b1, a.m);
    const int64_t rows = (int64_t)tk.n * a.group;
    len = max(len, 0);
    const int32_t cached = (int32_t)min((int64_t)len, (int64_t)a.max_pages << a.shift);
    const int64_t head_bytes = (int64_t)HD << a.shift, page_bytes = 2 * a.n_kv * head_bytes;
    const int8_t *keys = a.cache + kv * head_bytes, *values = keys + a.n_kv * head_bytes;

    for (int64_t tile = tile0; tile * 16 < rows; tile += a.tiles) {
        const bool whole = a.splits == 1 || tile >= a.tiles;  // this workgroup alone sees all keys
        if (whole && split) continue;
        // row r: token i, head of the group
        const int32_t i0 = tile ? (int32_t)by_group(a, tile * 16) : 0, g0 = (int32_t)(tile * 16 - (int64_t)i0 * a.group) + r;
        const bool real = tile * 16 + r < rows;
        const int32_t di = a.group >= 16 ? (g0 >= a.group ? 1 : 0) : (int32_t)(((float)g0 + 0.5f) * a.inv_group);  // (g0 < 32)
        const int32_t i = i0 + di, head = kv * a.group + (g0 - di * a.group);
        // (a tile's queries see no more keys than its last one, lane 15's or the last real one's; lanes without a query see
        // as many, so that spans seen whole need no masks)
        const int32_t last = min(__builtin_amdgcn_readlane(i, 15), tk.n - 1);
        const int32_t most = a.causal ? min(len - tk.n + last + 1, cached) : cached;
        const int32_t limit = real && a.causal ? min(len - tk.n + i + 1, cached) : most;
        const int32_t k0 = whole ? 0 : split * a.split_keys;
        const int32_t k1 = whole || split == a.splits - 1 ? most : min(most, k0 + a.split_keys);
        if (!whole && k0 >= most && split) continue;  // (part 0 says that there is none)

        i32x4 q[N];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            q[n] = i32x4{0, 0, 0, 0};
            if (real && 64 * n + 16 * h < HD)
                q[n] = *reinterpret_cast<const i32x4 *>(
                    a.q + at((int64_t)tk.first + i, head * HD + 64 * n + 16 * h, a.q_cols, a.q_cb));
        }
        f32x4 o[F];
#pragma unroll
        for (int f = 0; f < F; ++f) o[f] = f32x4{0, 0, 0, 0};
        float l = 0.0f;
        int32_t m = kNone;

        const int32_t kb0 = k0 + wave * kSpan;
        if (kb0 < k1 && tile != tile0) entries(kb0);
        for (int32_t kb = kb0; kb < k1; kb += kWaves * kSpan) {
            // key 16 (x / 4) + 4 t + x % 4 of the span is row x of score tile t, so that a lane's scores are those of
            // the 16 keys whose values it takes
            i32x4 kr[4][N], vr[F];
            {
                const int32_t page = (uint32_t)pk < (uint32_t)a.n_pages ? pk : 0;
                const int8_t *from = keys + page * page_bytes + (((kb + 16 * (r >> 2)) & in_mask) + (r & 3)) * HD;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        kr[t][n] = *reinterpret_cast<const i32x4 *>(from + 4 * t * HD + (64 * n + 16 * h < HD ? 64 * n + 16 * h : 0));
            }
            const bool there = (uint32_t)pv < (uint32_t)a.n_pages;
            {
                const int32_t page = there ? pv : 0;
                const int8_t *from = values + page * page_bytes + (((kb + 16 * h) & in_mask) * HD + r * 16);
#pragma unroll
                for (int f = 0; f < F; ++f) vr[f] = *reinterpret_cast<const i32x4 *>(from + 256 * f);
            }
            const int32_t seen = there ? limit - (kb + 16 * h) : 0;  // of the lane's 16 keys, those that its query sees
            entries(kb + kWaves * kSpan);
            asm volatile("" ::: "memory");
            i32x4 s[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                s[t] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int n = 0; n < N; ++n) s[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kr[t][n], q[n], s[t], 0, 0, 0);
            }
            int32_t top = kNone;
            const bool full = __all(seen >= 16);
            if (!full) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (4 * t + e >= seen) s[t][e] = kNone;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max(top, s[t][e]);
            top = quad_max(top);
            uint32_t sum = 0;
            i32x4 d0, d1, d2;
            const auto weights = [&](auto masked) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float p = __builtin_amdgcn_exp2f((float)(s[t][e] - top) * a.c2);
                        if (masked && 4 * t + e >= seen) p = 0.0f;  // (with a c2 of 0 too)
                        w[e] = __float_as_uint(fmaf(p, kLargest, kDigits));
                        sum += w[e];
                    }
                    const uint32_t low01 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u);
                    const uint32_t low23 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
                    const uint32_t top01 = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0602u);
                    const uint32_t top23 = __builtin_amdgcn_perm(w[3], w[2], 0x0c0c0602u);
                    d0[t] = (int)(__builtin_amdgcn_perm(low23, low01, 0x05040100u) ^ 0x80808080u);
                    d1[t] = (int)(__builtin_amdgcn_perm(low23, low01, 0x07060302u) ^ 0x80808080u);
                    d2[t] = (int)__builtin_amdgcn_perm(top23, top01, 0x05040100u);
                }
                sum -= 16 * kDigitsBits;  // (of 2^32: the sum itself is below)
            };
            if (full)
                weights(std::false_type{});
            else
                weights(std::true_type{});
            const int32_t now = max(m, top);
            const float fo = __builtin_amdgcn_exp2f((float)(m - now) * a.c2);
            const float fb = __builtin_amdgcn_exp2f((float)(top - now) * a.c2);
            m = now;
            l = l * fo + fb * (float)sum;
            // (two tiles of features at a time: all at once, their sums would take 12 F registers)
#pragma unroll
            for (int f0 = 0; f0 < F; f0 += FB) {
                i32x4 c0[FB], c1[FB], c2[FB];
#pragma unroll
                for (int j = 0; j < FB; ++j) {
                    if (f0 + j >= F) continue;
                    const i32x4 none = {0, 0, 0, 0};
                    c0[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vr[f0 + j], d0, none, 0, 0, 0);
                    c1[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vr[f0 + j], d1, none, 0, 0, 0);
                    c2[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vr[f0 + j], d2, none, 0, 0, 0);
                }
#pragma unroll
                for (int j = 0; j < FB; ++j) {
                    if (f0 + j >= F) continue;
                    f32x4 &to = o[f0 + j];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = fmaf((float)c2[j][e], 65536.0f, (float)(c1[j][e] * 256 + c0[j][e]));
                        to[e] = to[e] * fo + v * fb;
                    }
                    asm volatile("" : "+v"(to));
                }
                if (f0 + FB < F) asm volatile("" : "+v"(vr[f0 + FB]));  // (the next ones' products after this)
            }
        }
        // the waves' m, l and O together
        l = quad_sum(l);
        if (h == 0) {
            ms[wave][r] = m;
            ls[wave][r] = l;
        }
        __syncthreads();
        int32_t mm = ms[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) mm = max(mm, ms[w][r]);
        const float fw = __builtin_amdgcn_exp2f((float)(m - mm) * a.c2);
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) parts[wave][4 * f + e][lane] = o[f][e] * fw;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += ls[w][r] * __builtin_amdgcn_exp2f((float)(ms[w][r] - mm) * a.c2);
        __syncthreads();
        float *rec = whole ? nullptr
                           : a.work + ((((int64_t)seq * a.n_kv + kv) * a.tiles + tile) * a.splits + split) * record(HD, 16);
        if (rec && wave == 0 && h == 0) {
            reinterpret_cast<int32_t *>(rec)[r] = mm;
            rec[16 + r] = sum;
        }
        for (int f = wave; f < F; f += kWaves) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = parts[0][4 * f + e][lane];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) v[e] += parts[w][4 * f + e][lane];
            }
            if (!real) continue;
            if (rec)
                *reinterpret_cast<f32x4 *>(rec + 32 + r * HD + 16 * f + 4 * h) = v;
            else
                store_row(a, (int64_t)tk.first + i, head, 16 * f + 4 * h, v, sum);
        }
        __syncthreads();
    }
}

// The parts of a query together: join_group threads of 4 features each take every join_group-th part, and meet in LDS.
__global__ __launch_bounds__(256) void cache_join_kernel(const CacheArgs a)
{
    __shared__ __attribute__((aligned(16))) float sums[256][4];
    __shared__ float ls[256];
    __shared__ int32_t ms[256];
    const int tid = threadIdx.x;
    const int32_t seq = a.seq0 + blockIdx.y;
    const int32_t kv = a.tiles == 1 ? blockIdx.x : blockIdx.x / (uint32_t)a.tiles, tile = blockIdx.x - kv * a.tiles;
    int32_t b0 = ((ScalarTable)(uintptr_t)a.seq_start)[seq], b1 = ((ScalarTable)(uintptr_t)a.seq_start)[seq + 1];
    int32_t len = ((ScalarTable)(uintptr_t)a.kv_len)[seq];
    asm volatile("" : "+s"(b0), "+s"(b1), "+s"(len));  // (here they are all waited for, instead of one after the other)
    const Tokens tk = tokens_between(b0, b1, a.m);
    const int64_t first_row = (int64_t)tile * a.tile_rows;
    const int64_t rows = min((int64_t)tk.n * a.group - first_row, (int64_t)a.tile_rows);
    if (rows <= 0) return;
    len = max(len, 0);
    const int32_t cached = (int32_t)min((int64_t)len, (int64_t)a.max_pages << a.shift);
    const int32_t most = a.causal ? min(len - tk.n + (int32_t)by_group(a, first_row + rows - 1) + 1, cached) : cached;
    const int32_t n = min(a.splits, (max(most, 1) - 1) / a.split_keys + 1);  // (a part's keys more may not fit)
    const float *rec = a.work + (((int64_t)seq * a.n_kv + kv) * a.tiles + tile) * a.splits * record(a.hd, a.tile_rows);
    const int quads = a.hd / 4, per = quads * a.join_group, here_rows = 256 / per;  // rows of a workgroup at a time
    const int mine = tid / per, group = tid % per / quads, c = tid % quads * 4;
    // (as many workgroups as a tile was said to have rows; a sequence with more tokens than that has more)
    for (int r0 = blockIdx.z * here_rows; r0 < rows; r0 += gridDim.z * here_rows) {
        const int r = r0 + mine;
        const bool real = mine < here_rows && r < rows;
        int32_t m = kNone;
        float l = 0.0f;
        f32x4 o = {0, 0, 0, 0};
        for (int s0 = group; s0 < n && real; s0 += 4 * a.join_group) {
            int32_t mp[4];
            float lp[4];
            f32x4 op[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int s = s0 + j * a.join_group;
                const float *p = rec + (int64_t)min(s, n - 1) * record(a.hd, a.tile_rows);
                mp[j] = s < n ? reinterpret_cast<const int32_t *>(p)[r] : kNone;
                lp[j] = s < n ? p[a.tile_rows + r] : 0.0f;
                op[j] = *reinterpret_cast<const f32x4 *>(p + 2 * a.tile_rows + r * a.hd + c);
            }
            const int32_t now = max(max(max(mp[0], mp[1]), max(mp[2], mp[3])), m);
            const float f = __builtin_amdgcn_exp2f((float)(m - now) * a.c2);
            l *= f;
            o *= f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float g = s0 + j * a.join_group < n ? __builtin_amdgcn_exp2f((float)(mp[j] - now) * a.c2) : 0.0f;
                l += lp[j] * g;
                o += op[j] * g;
            }
            m = now;
        }
        if (a.join_group > 1) {
            ms[tid] = m;
            ls[tid] = l;
            *reinterpret_cast<f32x4 *>(sums[tid]) = o;
            __syncthreads();
            if (group == 0 && real) {
                int32_t mm = m;
                for (int g = 1; g < a.join_group; ++g) mm = max(mm, ms[tid + g * quads]);
                l = 0.0f;
                o = f32x4{0, 0, 0, 0};
                for (int g = 0; g < a.join_group; ++g) {
                    const float f = __builtin_amdgcn_exp2f((float)(ms[tid + g * quads] - mm) * a.c2);
                    l += ls[tid + g * quads] * f;
                    o += *reinterpret_cast<const f32x4 *>(sums[tid + g * quads]) * f;
                }
            }
            __syncthreads();
        }
        if (group == 0 && real) {
            const int64_t row = first_row + r;
            const int32_t i = (int32_t)by_group(a, row);
            store_row(a, (int64_t)tk.first + i, kv * a.group + (int32_t)(row - (int64_t)i * a.group), c, o, l);
        }
    }
}

template <int F>
sl_status launch_split(const CacheArgs &a, dim3 grid, hipStream_t s)
{
    if (a.by_length)
        hipLaunchKernelGGL((cache_split_kernel<F, true>), grid, dim3(64 * kWaves), 0, s, a);
    else
        hipLaunchKernelGGL((cache_split_kernel<F, false>), grid, dim3(64 * kWaves), 0, s, a);
    HIP_TRY(hipGetLastError());
    return SL_OK;
}

}  // namespace

int64_t cache_attention_bytes(const sl_cache_attention_args &a)
{
    const AttentionPlan p = plan_of(a);
    if (p.splits == 1) return 0;
    return (int64_t)a.n_seq * a.n_kv_heads * p.tiles * p.splits * record(a.head_dim, p.tile_rows) * 4;
}

sl_status launch_cache_append(const sl_cache_append_args &a, void *stream)
{
    const AppendPlan plan = plan_of(a);
    if (!plan.fits) {
        set_error("too many work items for one launch");
        return SL_ERR_UNSUPPORTED;
    }
    const bool f32 = a.x_type == SL_ACT_F32;
    AppendArgs p{};
    p.x = static_cast<const int8_t *>(a.x);
    p.q = a.q;
    p.cache = a.cache;
    p.seq_start = a.seq_start;
    p.kv_len = a.kv_len;
    p.page_table = a.page_table;
    p.positions = a.positions;
    p.inv_freq = a.inv_freq;
    p.m = a.m_tokens;
    p.max_pages = a.max_pages;
    p.n_pages = a.n_pages;
    p.shift = __builtin_ctz(a.page_size);
    p.nh = a.n_heads;
    p.nkv = a.n_kv_heads;
    p.hd = a.head_dim;
    const int32_t cols = (a.n_heads + 2 * a.n_kv_heads) * a.head_dim;
    p.x_cb = !f32 && a.x_layout == SL_LAYOUT_T16X32 ? (cols + 31) / 32 : 0;
    p.q_cb = a.q_layout == SL_LAYOUT_T16X32 ? (a.n_heads * a.head_dim + 31) / 32 : 0;
    p.x_step = p.x_cb ? p.x_cb * 512 : cols * (f32 ? 4 : 1);
    p.q_step = p.q_cb ? p.q_cb * 512 : a.n_heads * a.head_dim;
    p.values = (uint32_t)(a.n_kv_heads * a.head_dim) << p.shift;
    p.page_bytes = 2 * (int64_t)p.values;
    p.half = a.rope_kind != SL_ROPE_NONE ? a.rope_dim / 2 : 0;
    p.split = a.rope_kind == SL_ROPE_HALF;
    p.rope_factor = a.rope_factor;
    // (finite, so that 0 stays 0; what it cuts is a code of 127 all the same)
    const auto factor = [&](float scale) {
        return std::min(f32 ? 1.0f / scale : (float)std::min((double)a.x_scale / scale, (double)FLT_MAX), FLT_MAX);
    };
    p.fq = factor(a.q_scale);
    p.fk = factor(a.k_scale);
    p.fv = factor(a.v_scale);
    p.q_columns = plan.q_columns;
    p.k_columns = plan.k_columns;
    p.v_columns = plan.v_columns;
    p.q_parts = plan.q_parts;
    p.k_parts = plan.k_parts;
    p.per = plan.per;
    p.v_per = plan.v_per;
    const int32_t width = plan.vec ? 8 : 2;
    p.inv_qk = (float)width / a.head_dim;
    p.inv_value = 4.0f / a.head_dim;
    p.inv_half = p.half ? 1.0f / p.half : 0.0f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    for (int64_t s0 = 0; s0 < a.n_seq; s0 += kMostGrid) {
        p.seq0 = (int32_t)s0;
        const dim3 grid((uint32_t)plan.parts, (uint32_t)plan.groups, (uint32_t)std::min(a.n_seq - p.seq0, kMostGrid));
        const auto run = [&](auto types, auto widths) {
            constexpr bool F = decltype(types)::value, V = decltype(widths)::value;
            if (plan.step)
                hipLaunchKernelGGL((cache_append_step_kernel<F, V>), grid, dim3(256), 0, s, p);
            else
                hipLaunchKernelGGL((cache_append_kernel<F, V>), grid, dim3(256), 0, s, p);
        };
        if (f32 && plan.vec)
            run(std::true_type{}, std::true_type{});
        else if (f32)
            run(std::true_type{}, std::false_type{});
        else if (plan.vec)
            run(std::false_type{}, std::true_type{});
        else
            run(std::false_type{}, std::false_type{});
        HIP_TRY(hipGetLastError());
    }
    return SL_OK;
}

sl_status launch_cache_attention(const sl_cache_attention_args &args, void *stream)
{
    CacheArgs a{};
    a.q = args.q;
    a.cache = args.cache;
    a.seq_start = args.seq_start;
    a.kv_len = args.kv_len;
    a.page_table = args.page_table;
    a.y = args.y;
    a.work = static_cast<float *>(args.workspace);
    a.m = args.m_tokens;
    const AttentionPlan p = plan_of(args);
    if (!p.fits) {
        set_error("too many work items for one launch");
        return SL_ERR_UNSUPPORTED;
    }
    a.n_seq = args.n_seq;
    a.tiles = p.tiles;
    a.splits = p.splits;
    a.split_keys = p.split_keys;
    a.n_heads = args.n_heads;
    a.n_kv = args.n_kv_heads;
    a.group = args.n_heads / args.n_kv_heads;
    a.hd = args.head_dim;
    a.q_cols = args.q_cols;
    a.q_cb = args.q_layout == SL_LAYOUT_T16X32 ? (args.q_cols + 31) / 32 : 0;
    a.y_cb = args.y_layout == SL_LAYOUT_T16X32 ? (args.n_heads * args.head_dim + 31) / 32 : 0;
    a.shift = __builtin_ctz(args.page_size);
    a.max_pages = args.n_pages ? args.max_pages : 0;  // (no page: nothing is read)
    a.n_pages = args.n_pages;
    a.causal = args.causal;
    a.y_f32 = args.kind == SL_EPI_F32;
    a.c2 = (float)((double)args.q_scale * args.k_scale * args.softmax_scale * 1.4426950408889634);
    // A result is a mean of codes (vs / l times their sum) times `unit`, where vs is v_scale's mantissa, 1 .. 2, and unit has
    // its exponent: v_scale / l may be less than a float holds in full, and v_scale / out_scale more than one.
    int ev = 0, eo = 0;
    a.vs = 2.0f * frexpf(args.v_scale, &ev);
    const float mo = a.y_f32 ? 1.0f : 2.0f * frexpf(args.out_scale, &eo);
    a.unit = (float)std::min(ldexp((double)(1.0f / mo), a.y_f32 ? ev - 1 : ev - eo), a.y_f32 ? (double)FLT_MAX : (double)FLT_MAX / 4);
    a.inv_group = 1.0f / a.group;
    a.group_shift = (a.group & (a.group - 1)) ? -1 : __builtin_ctz(a.group);
    a.tile_rows = p.tile_rows;
    a.by_length = p.by_length;
    if (p.prompt) {
        const Exponent e = exponent_of((double)args.q_scale * args.k_scale * args.softmax_scale);
        a.c2 = e.c2;
        a.k2 = e.k2;
    }
    // threads of a row's 4 features that share its parts, 4 and more each; and workgroups for a tile's rows
    const int32_t quads = a.hd / 4;
    a.join_group = std::min(256 / quads, (a.splits + 3) / 4);
    const int32_t at_a_time = 256 / (quads * a.join_group);
    const int32_t join_z = (int32_t)((std::min<int64_t>(a.tile_rows, (int64_t)args.max_new * a.group) + at_a_time - 1) / at_a_time);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    for (int64_t s0 = 0; s0 < a.n_seq; s0 += kMostGrid) {
        a.seq0 = (int32_t)s0;
        const uint32_t seqs = (uint32_t)std::min(a.n_seq - a.seq0, kMostGrid);
        const dim3 grid((uint32_t)(a.n_kv * a.tiles), seqs, (uint32_t)a.splits);
        sl_status st = SL_OK;
        switch (p.prompt ? 0 : a.hd / 16) {
        case 0: st = launch_cache_prompt(a, dim3((uint32_t)a.n_kv, seqs, (uint32_t)(a.tiles * a.splits)), s); break;
        case 1: st = launch_split<1>(a, grid, s); break;
        case 2: st = launch_split<2>(a, grid, s); break;
        case 3: st = launch_split<3>(a, grid, s); break;
        case 4: st = launch_split<4>(a, grid, s); break;
        case 5: st = launch_split<5>(a, grid, s); break;
        case 6: st = launch_split<6>(a, grid, s); break;
        case 7: st = launch_split<7>(a, grid, s); break;
        default: st = launch_split<8>(a, grid, s); break;
        }
        if (st != SL_OK) return st;
        if (a.splits > 1) {
            hipLaunchKernelGGL(cache_join_kernel, dim3(grid.x, seqs, (uint32_t)join_z), dim3(256), 0, s, a);
            HIP_TRY(hipGetLastError());
        }
    }
    // (numbers put down by hand: formatting them is a part of what a short call costs)
    char name[40] = "";
    char *end = name + sizeof(name) - 1, *at = name;
    for (const char *c = p.prompt ? "cache prompt " : "cache split "; *c; ++c) *at++ = *c;
    at = std::to_chars(at, end, a.hd).ptr;
    *at++ = ',';
    *std::to_chars(at, end, a.splits).ptr = 0;
    set_last_path("%s", name);
    return SL_OK;
}

}  // namespace sl
