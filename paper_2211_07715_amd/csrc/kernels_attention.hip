// attention_run and attention_select (gfx950).
//
// Attention. For one head and a tile of queries, over chunks of 64 keys:
//   S = K Q^T            int8 x int8 -> int32 on v_mfma_i32_32x32x32_i8, exact
//   P = 2^(c (S - m))    m: about the largest of a query's S
//   l += sum P, O += V^T P^T   on v_mfma_f32_32x32x16_f16
// and y = x_scale O / l. S is computed transposed (keys are the matrix
// instruction's rows, queries its columns), so that a lane's scores all belong
// to one query and lie where the second product takes its right operand from:
// lane half h of a 32-key tile holds keys 8 i + 4 h .. 8 i + 4 h + 3, and its 8
// scores of 16 keys, rounded to 16 bits, are the 8 values a lane gives to a
// 16-key product. That product may take the keys in any order as long as V's
// operand has them in the same one, so V is laid out in LDS in that order.
//
// The integer scores meet the exponential without a conversion: the
// accumulators start at the bits of 1.5 * 2^23 as a float, less m, so that the
// finished sums read as floats are 1.5 * 2^23 + (S - m) exactly
// (|S - m| <= 2^22 for heads of up to 128 features), and one fused multiply-add
// gives the exponent.
//
// What bounds it: the vector instructions (an exponential 8.3 cycles of a SIMD,
// a conversion, permute or dot product 4.3, a fused multiply-add 2.6) with one
// tile of queries a wave; with two, which stage a chunk half as often, vector and
// matrix instructions together, which overlap only in part. 32 x 32 matrix ones
// take less of the issue than 16 x 16 ones of the same work. m may lag behind the
// running maximum by a factor of 2^8, which 16-bit P leaves room for: it moves,
// and l and O are rescaled, outside the loop over chunks, which is left for that
// and entered again (a branch inside would make the compiler copy every
// accumulator).
//
// Measured, 4 operations a score and feature, replayed from a graph: 128 x 384
// tokens of 12 heads of 64 111 us (522 TOP/s), 8192 tokens of 16 heads on 4 367 us
// (749 TOP/s), 32 blocks at 16384 tokens of 12 heads 171 us (603 TOP/s), 32 x 128
// tokens 9.0 us, 128 tokens 6.5 us. In traced launches of the same three long
// cases (110, 431 and 187 us) vector instructions are active up to 86, 73 and 77
// % of the time (counted in steps of 4 cycles, more than a plain one takes),
// and matrix ones run 35, 43 and 36 %.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <string>

#include "attention_device.h"
#include "encoder.h"

namespace sl {

namespace {

typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
typedef int16_t i16x8 __attribute__((ext_vector_type(8)));
struct AttnArgs {
    const int8_t *x;
    const int32_t *seq_start, *key_len, *blocks;
    void *y;
    int64_t m;
    int64_t n_items;
    int32_t n_seq, tiles, tq, n_heads, n_kv, hd, cols, x_cb, y_cb;
    int32_t top_k, n_qb, halvings, y_f32;  // tq << halvings: queries of a list
    float c2, k2, inv_so, xs;
};

// tokens first .. first + n - 1 of a sequence and its valid keys
struct Span {
    int32_t first, n, keys;
};
__device__ __forceinline__ Span span_of(const int32_t *seq_start, const int32_t *key_len, int32_t s, int64_t m)
{
    const int32_t m32 = (int32_t)m;
    const int32_t b = min(max(seq_start[s], 0), m32), e = min(max(seq_start[s + 1], b), m32);
    const int32_t n = e - b;
    return {b, n, key_len ? min(max(key_len[s], 0), n) : n};
}

// 4 keys x 4 features of int8 (words k0 .. k3, a byte a feature) as 16-bit
// floats, feature by feature. A code c as an unsigned byte u = c + 128 under
// the byte 0x64 is the 16-bit float 1024 + u; 1152 less is c, exactly.
__device__ __forceinline__ void transpose_to_f16(const uint32_t (&k)[4], u32x2 (&out)[4])
{
    const uint32_t f = 0x80808080u, e = 0x64646464u;
    const uint32_t a = k[0] ^ f, b = k[1] ^ f, c = k[2] ^ f, d = k[3] ^ f;
    // bytes: a0 b0 a1 b1, a2 b2 a3 b3 and the same of c, d
    const uint32_t ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u), ab2 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t cd0 = __builtin_amdgcn_perm(d, c, 0x05010400u), cd2 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
    const auto low = [&](uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(e, w, 0x04010400u)) - bias);
    };
    const auto high = [&](uint32_t w) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(e, w, 0x04030402u)) - bias);
    };
    out[0] = {low(ab0), low(cd0)};
    out[1] = {high(ab0), high(cd0)};
    out[2] = {low(ab2), low(cd2)};
    out[3] = {high(ab2), high(cd2)};
}

// Where a thread's pieces of a chunk lie: bytes from the chunk's first token's
// row block. Both layouts advance by a constant from chunk to chunk, so a
// thread's offsets are computed once.
struct Rows {
    const int8_t *base;  // of the sequence (block layout: of the 16-token block of its first token)
    int32_t skip;        // block layout: tokens of that block before it
    int32_t cols, cb;
    int64_t chunk;       // bytes from a chunk to the next
    __device__ __forceinline__ Rows(const int8_t *x, int32_t first, int32_t cols_, int32_t cb_)
        : cols(cols_), cb(cb_)
    {
        skip = cb ? first & 15 : 0;
        base = cb ? x + (int64_t)(first >> 4) * cb * 512 : x + (int64_t)first * cols;
        chunk = cb ? (int64_t)(kChunk / 16) * cb * 512 : (int64_t)kChunk * cols;
    }
    // row `key` (less than 2 chunks) and feature c
    __device__ __forceinline__ uint32_t offset(int32_t key, int32_t c) const
    {
        const int32_t t = key + skip;
        return cb ? (uint32_t)((t >> 4) * cb + (c >> 5)) * 512 + (t & 15) * 32 + (c & 31) : (uint32_t)(key * cols + c);
    }
};

// N: 32-feature tiles of a head (head_dim <= 32 N); NW: waves, of QT tiles of 32
// queries each, which share the chunk of keys and values in LDS. Two
// buffers: while one chunk is multiplied, the next one's K is loaded into the
// other buffer and its V into registers, which are written there (transposed)
// before the barrier. That K takes no registers lets lists of 64 queries have
// three waves a SIMD: 32 blocks at 16384 tokens of 12 heads 185 us against 211.
// One wave has one buffer and K in registers (twice the workgroups in LDS: 16
// blocks at 8192 tokens of 12 heads, query_block 32, 66 us against 72).
//
// SPLIT > 1 (NW is 1 then): a workgroup is SPLIT waves on the same queries, each
// with every SPLIT-th chunk in a buffer of its own and no barrier until their m,
// l and O meet in LDS at the end.
//
// At most 256 registers (two waves a SIMD; three for the shape of most calls), so
// that the accumulators are ordinary registers, which the exponentials read
// without a copy. One wave that brings in whole chunks of a head of more than 64
// features takes more (one wave a SIMD).
template <int N, int QT, int NW, int SPLIT, bool LISTS>
__global__ __launch_bounds__(64 * NW * SPLIT)
__attribute__((amdgpu_waves_per_eu(N <= 2 && QT == 1 && NW >= 2 ? 3 : N > 2 && NW == 1 ? 1 : 2)))
void attention_kernel(const AttnArgs a)
{
    constexpr int D = 32 * N;
    constexpr int VS = 2 * kChunk;             // LDS bytes of a feature of V (of a key: D)
    constexpr int KB = kChunk * D, BUF = KB + D * VS;
    constexpr int NT = 64 * NW;
    constexpr int KN = kChunk * 2 * N, VN = kChunk / 4 * D / 4;  // a chunk's 16-byte pieces of K and 4 x 4 ones of V
    constexpr int KP = (KN + NT - 1) / NT, VP = (VN + NT - 1) / NT;  // and a thread's
    constexpr int NBUF = NW > 1 ? 2 : 1;  // (one wave's reads and writes of LDS keep their order)
    static_assert(SPLIT == 1 || (NW == 1 && QT == 1), "one wave a part");
    constexpr bool DIRECT = NBUF > 1;  // K goes to LDS without registers
    // (the parts' O: 16 N floats a lane)
    constexpr int LDS = SPLIT * std::max(NBUF * BUF, SPLIT > 1 ? 64 * 64 * N : 0);
    __shared__ __attribute__((aligned(16))) char all_lds[LDS];
    const int tid = threadIdx.x % NT, lane = tid & 63, wave = tid >> 6, half = lane >> 5, n32 = lane & 31;
    const int part = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    char *lds = all_lds + part * (NBUF * BUF);
    const auto sync = [] {
        if constexpr (NW > 1)
            __syncthreads();
        else
            asm volatile("" ::: "memory");
    };
    const uint32_t item = (uint32_t)xcd_work_index(blockIdx.x, a.n_items);
    const int32_t tile = (int32_t)(item % (uint32_t)a.tiles);
    const int32_t head = (int32_t)(item / (uint32_t)a.tiles % (uint32_t)a.n_heads);
    const int32_t seq = (int32_t)(item / (uint32_t)a.tiles / (uint32_t)a.n_heads);
    const Span sp = span_of(a.seq_start, a.key_len, seq, a.m);
    if ((int64_t)tile * a.tq >= sp.n) return;
    const int32_t kv = head / (a.n_heads / a.n_kv);
    const int32_t kcol = (a.n_heads + kv) * a.hd, vcol = (a.n_heads + a.n_kv + kv) * a.hd;
    const Rows rows(a.x, sp.first, a.cols, a.x_cb);

    // A thread's pieces: key and feature of K piece i, first key and feature of
    // V piece i. Features past the head's are read as its first ones (they meet
    // zeros of Q, or give sums that are not stored), keys past a short chunk's
    // as its last one (their weights are zero).
    const auto kpiece = [&](int i, int &key, int &d) {
        const int p = tid + i * NT;
        key = p / (2 * N) % kChunk;
        d = (p % (2 * N) ^ (DIRECT ? kswap<N>(key) : 0)) * 16;
    };
    const auto vpiece = [&](int i, int &key, int &d) {
        const int p = tid + i * NT;  // (8 lanes: 32 keys of 4 features, whose stores fill 64 bytes of LDS)
        key = (p % 8 + p / (2 * D) * 8) % (kChunk / 4) * 4;
        d = p / 8 % (D / 4) * 4;
    };
    uint32_t koff[KP], voff[VP][4], kdst[KP], vdst[VP];
    const auto offsets = [&](int32_t have) {
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            int key, d;
            kpiece(i, key, d);
            koff[i] = rows.offset(min(key, have - 1), kcol + (d < a.hd ? d : 0));
        }
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            int key, d;
            vpiece(i, key, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) voff[i][j] = rows.offset(min(key + j, have - 1), vcol + (d < a.hd ? d : 0));
        }
    };
#pragma unroll
    for (int i = 0; i < KP; ++i) {
        int key, d;
        kpiece(i, key, d);
        kdst[i] = key * D + 16 * (d / 16 ^ kswap<N>(key));
    }
#pragma unroll
    for (int i = 0; i < VP; ++i) {
        int key, d;
        vpiece(i, key, d);
        // place of keys 4 q .. 4 q + 3 of 16 in a feature's row: their lane half's 8, first or second 4
        const int q = key / 4, pos = (q >> 2) * 16 + (q & 1) * 8 + ((q >> 1) & 1) * 4;
        // row of a feature: lane half h of a tile's rows 8 x + 4 h + b then holds features 16 N h + 16 tile + 4 x + b
        const int row = 32 * (d / 16 % N) + 8 * (d / 4 % 4) + 4 * (d / (16 * N));
        vdst[i] = KB + row * VS + ((2 * pos) ^ (16 * vswap(row)));
    }
    i32x4 kreg[KP];
    uint32_t vreg[VP][4];
    // Where a thread's pieces are the same features of keys KSTEP (V: 32) apart, one offset serves them in a whole chunk.
    constexpr int KSTEP = NT % (2 * N) == 0 && NT / (2 * N) % 16 == 0 ? NT / (2 * N) : 0;
    constexpr bool VHALF = VP == 2 && NT == 2 * D;
    const int32_t group = rows.cb ? rows.cb * 512 : 16 * rows.cols;  // bytes of 16 keys
    const auto load = [&](int32_t b, bool full, char *buf) __attribute__((always_inline)) {
        // (the offsets are in bounds: the resource only spares the lanes 64-bit addresses)
        const auto x = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(rows.base + b * rows.chunk), 0, 0x7fffffff,
                                                         kRsrcWord3);
#pragma unroll
        for (int i = 0; i < KP; ++i) {
            const bool step = KSTEP && full;
            const int32_t more = step ? i * (KSTEP / 16) * group : 0;
            const int first = __builtin_amdgcn_readfirstlane(tid) + i * NT;
            if constexpr (DIRECT) {
                if (KP * NT == KN || first < KN)
                    load_to_lds(x, buf + 16 * first, koff[step ? 0 : i], more);
            } else {
                kreg[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(x, koff[step ? 0 : i], more, 0));
            }
        }
#pragma unroll
        for (int i = 0; i < VP; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool step = VHALF && full;
                vreg[i][j] = __builtin_amdgcn_raw_buffer_load_b32(x, voff[step ? 0 : i][j], step ? i * 2 * group : 0, 0);
            }
    };
    const auto stage = [&](char *buf) {
#pragma unroll
        for (int i = 0; i < KP; ++i)
            if (!DIRECT && (KP * NT == KN || tid + i * NT < KN)) *reinterpret_cast<i32x4 *>(buf + (KSTEP ? kdst[0] + i * KSTEP * D : kdst[i])) = kreg[i];
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            if (VP * NT == VN || tid + i * NT < VN) {
                u32x2 out[4];
                transpose_to_f16(vreg[i], out);
                // (of rows 4 x .. 4 x + 3, the last two have the lowest bit of the swap set)
                const uint32_t dst = VHALF ? vdst[0] ^ (64 * i) : vdst[i];
                char *to = buf + dst, *to2 = buf + (dst ^ 16);
                *reinterpret_cast<u32x2 *>(to) = out[0];
                *reinterpret_cast<u32x2 *>(to + VS) = out[1];
                *reinterpret_cast<u32x2 *>(to2 + 2 * VS) = out[2];
                *reinterpret_cast<u32x2 *>(to2 + 3 * VS) = out[3];
            }
        }
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };

    for (int32_t qt = tile; (int64_t)qt * a.tq < sp.n; qt += a.tiles) {
        // a lane's query of tile t; past the queries of the sequence or of a small query block, none
        const auto query = [&](int t) {
            const int32_t i = (wave * QT + t) * 32 + here(n32), qi = qt * a.tq + i;
            return i < a.tq && qi < sp.n ? qi : -1;
        };
        i32x4 q[QT][N];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int32_t qi = query(t);
#pragma unroll
            for (int h = 0; h < N; ++h) {
                const int32_t d = 32 * h + 16 * here(half);
                q[t][h] = i32x4{0, 0, 0, 0};
                if (qi >= 0 && d < a.hd)
                    q[t][h] = *reinterpret_cast<const i32x4 *>(
                        a.x + at((int64_t)sp.first + qi, head * a.hd + d, a.cols, a.x_cb));
            }
        }
        f32x16 o[QT][N];
        float l[QT];
        int32_t z[QT];  // what S starts at: kMagic - m
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            l[t] = 0.0f;
            z[t] = kMagic - kLowest;
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][d][i] = 0.0f;
        }

        // scores of a chunk
        const auto scores = [&](int t, const char *buf, const i32x16 &from, i32x16 (&s)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                s[kt] = from;
#pragma unroll
                for (int h = 0; h < N; ++h) {
                    const int row = 32 * kt + n32;
                    const i32x4 k = *reinterpret_cast<const i32x4 *>(buf + row * D + 16 * ((2 * h + half) ^ kswap<N>(n32)));
                    s[kt] = __builtin_amdgcn_mfma_i32_32x32x32_i8(k, q[t][h], s[kt], 0, 0, 0);
                }
            }
        };
        const auto from_z = [&](int t) {
            i32x16 v;
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = z[t];
            if constexpr (QT == 1) asm volatile("" : "+v"(v));  // 16 registers for the loop over chunks, not 32 moves in it
            return v;
        };
        // keys past the chunk's `have`: minus infinity, as the bits that the scores are
        const auto mask = [&](int32_t have, i32x16 (&s)[2]) __attribute__((always_inline)) {
            const int32_t mine = have - 4 * half;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * kt + 8 * (i / 4) + i % 4 >= mine) s[kt][i] = (int32_t)0xff800000;
        };
        // the largest of a lane's
        const auto largest = [&](const i32x16 (&s)[2]) __attribute__((always_inline)) {
            int32_t top = 0;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = max(top, s[kt][i]);
            return top;
        };
        // m up to the running maximum
        const auto raise = [&](int t, int32_t top) __attribute__((always_inline)) {
            const int32_t by = max(pair_max(top) - kMagic, 0);
            const float f = __builtin_amdgcn_exp2f(-(float)by * a.c2);
            z[t] -= by;
            l[t] *= f;
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][d][i] *= f;
        };
        // Weights of a chunk, in two 16-bit parts, and their sum. The first part is
        // the value cut to 11 bits, so the second is its remainder exactly: together
        // they hold 22, and a product with both costs matrix instructions, which
        // there is room for, where one of 11 bits changed 0.4 % of int8 results.
        // The remainder of a weight below 2^-10 of the largest is a subnormal of 16
        // bits: such weights are held to 2^-31 of the largest instead (the factor of
        // 2^7 that P carries included). The sum is that of the whole values.
        f16x8 p[QT][4], p2[QT][4];
        const auto weights = [&](int t, const i32x16 (&s)[2]) __attribute__((always_inline)) {
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {  // 16 keys
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    float e[2], hi[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int i = 8 * (w & 1) + j + r;
                        e[r] = __builtin_amdgcn_exp2f(fmaf(__int_as_float(s[w / 2][i]), a.c2, a.k2));
                        sum[2 * (w & 1) + r] += e[r];
                        hi[r] = __uint_as_float(__float_as_uint(e[r]) & 0xffffe000u);
                    }
                    const f16x2 h = __builtin_convertvector((f32x2{hi[0], hi[1]}), f16x2);
                    const f16x2 l2 = __builtin_convertvector((f32x2{e[0] - hi[0], e[1] - hi[1]}), f16x2);
                    p[t][w][j] = h[0];
                    p[t][w][j + 1] = h[1];
                    p2[t][w][j] = l2[0];
                    p2[t][w][j + 1] = l2[1];
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
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        o[t][d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[t][w], o[t][d], 0, 0, 0);
                        o[t][d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p2[t][w], o[t][d], 0, 0, 0);
                    }
                }
        };

        // Whole chunks first, then the sequence's short last one. With lists:
        // 64 numbers at a time, one a lane; those of whole chunks as a mask.
        const int32_t whole = sp.keys / kChunk, rest = sp.keys % kChunk;
        const int32_t steps = LISTS ? (qt >> a.halvings < a.n_qb ? a.top_k : 0) : whole;
        const int32_t *list =
            a.blocks + (((int64_t)seq * a.n_heads + head) * a.n_qb + (qt >> a.halvings)) * a.top_k;
        int32_t at_step = LISTS ? 0 : part, mine = -1, tails = !LISTS && rest && (SPLIT == 1 || whole % SPLIT == part);
        uint64_t left = 0;
        const uint64_t ours = SPLIT == 1 ? ~0ull : 0x1111111111111111ull << part;
        static_assert(SPLIT == 1 || SPLIT == 4, "every 4th of a list's numbers");
        const auto next = [&]() -> int32_t {  // the next whole chunk, or -1
            if constexpr (!LISTS) {
                const int32_t i = at_step;
                at_step += SPLIT;
                return i < steps ? i : -1;
            } else {
                while (!left) {
                    if (at_step >= steps) return -1;
                    mine = at_step + lane < steps ? list[at_step + lane] : -1;
                    left = __ballot((uint32_t)mine < (uint32_t)whole) & ours;
                    if (rest) tails += __popcll(__ballot(mine == whole) & ours);
                    at_step += 64;
                }
                const int i = __builtin_ctzll(left);
                left &= left - 1;
                return __builtin_amdgcn_readlane(mine, i);
            }
        };
        offsets(kChunk);
        i32x16 sc[2];
        int32_t b = next();
        if (b >= 0) {
            load(b, true, lds);
            stage(lds);
            b = next();
            sync();
            int32_t buf = 0;
            if (wave * 32 * QT >= a.tq) {  // a wave without queries only brings chunks in
                while (b >= 0) {
                    load(b, true, lds + (buf ^ BUF));
                    buf ^= BUF;
                    stage(lds + buf);
                    b = next();
                    sync();
                }
                goto done;
            }
            for (;;) {
                i32x16 from[QT];
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    scores(t, lds + buf, from_z(t), sc);
                    raise(t, largest(sc));
                    from[t] = from_z(t);
                }
                for (;;) {
                    if (b >= 0) load(b, true, lds + (buf ^ BUF));  // (again after m has moved)
                    float sum[QT];
                    bool over = false;  // (no weight is over 65504 while their sum is below kMostSum)
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        scores(t, lds + buf, from[t], sc);
                        sum[t] = weights(t, sc);
                        over |= !(sum[t] < kMostSum);
                    }
                    if (__any(over)) break;
#pragma unroll
                    for (int t = 0; t < QT; ++t) l[t] += sum[t];
                    multiply(lds + buf);
                    if (b < 0) goto done;
                    if constexpr (NBUF > 1) buf ^= BUF;
                    stage(lds + buf);
                    b = next();
                    sync();
                }
            }
        done:
            sync();
        }
        if (tails > 0) {
            offsets(rest);
            load(whole, false, lds);
            stage(lds);
            sync();
            for (int32_t i = 0; i < tails; ++i) {
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    scores(t, lds, from_z(t), sc);
                    mask(rest, sc);
                    raise(t, largest(sc));
                    scores(t, lds, from_z(t), sc);
                    mask(rest, sc);
                    l[t] += weights(t, sc);
                }
                multiply(lds);
            }
            sync();
        }
        if constexpr (SPLIT > 1) {
            // every part's l and O from the largest m; part w then sums registers 4 N w .. 4 N w + 4 N - 1 of all
            __shared__ int32_t zs[SPLIT][32];
            __shared__ float ls[SPLIT][32];
            l[0] = pair_sum(l[0]);
            __syncthreads();
            if (half == 0) {
                zs[part][n32] = z[0];
                ls[part][n32] = l[0];
            }
            __syncthreads();
            int32_t zmin = zs[0][n32];
#pragma unroll
            for (int w = 1; w < SPLIT; ++w) zmin = min(zmin, zs[w][n32]);
            const float f = __builtin_amdgcn_exp2f(-(float)(z[0] - zmin) * a.c2);
            float *mine_o = reinterpret_cast<float *>(all_lds) + part * (64 * 16 * N);
#pragma unroll
            for (int d = 0; d < N; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) mine_o[(16 * d + i) * 64 + lane] = o[0][d][i] * f;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < SPLIT; ++w)
                sum += ls[w][n32] * __builtin_amdgcn_exp2f(-(float)(zs[w][n32] - zmin) * a.c2);
            __syncthreads();
            const float g = sum > 0.0f ? a.xs / sum * (a.y_f32 ? 1.0f : a.inv_so) : 0.0f;
            const int32_t qi = query(0);
            const int64_t tok = (int64_t)sp.first + qi;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int first = 4 * N * part + 4 * i;
                f32x4 v = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < SPLIT; ++w)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        v[j] += reinterpret_cast<const float *>(all_lds)[w * (64 * 16 * N) + (first + j) * 64 + lane];
                const int32_t c = 16 * N * here(half) + first;
                if (qi < 0 || c >= a.hd) continue;
                if (a.y_f32)
                    *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.y) + tok * (a.n_heads * a.hd) + head * a.hd + c) = v * g;
                else
                    *reinterpret_cast<uint32_t *>(reinterpret_cast<int8_t *>(a.y) +
                                                  at(tok, head * a.hd + c, a.n_heads * a.hd, a.y_cb)) =
                        pack_bytes(requant_bits(v[0], g), requant_bits(v[1], g), requant_bits(v[2], g),
                                   requant_bits(v[3], g));
            }
            __syncthreads();
            continue;
        }
        // a lane half holds features 16 N half .. 16 N half + 16 N - 1 of its query
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float sum = pair_sum(l[t]);
            const float f = sum > 0.0f ? a.xs / sum * (a.y_f32 ? 1.0f : a.inv_so) : 0.0f;
            const int32_t qi = query(t);
            if (qi < 0) continue;
            const int64_t tok = (int64_t)sp.first + qi;
            const int h2 = here(half);
            if (a.y_f32) {
                float *y = reinterpret_cast<float *>(a.y) + tok * (a.n_heads * a.hd) + head * a.hd + 16 * N * h2;
#pragma unroll
                for (int d = 0; d < N; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        if (16 * N * h2 + 16 * d < a.hd)
                            *reinterpret_cast<f32x4 *>(y + 16 * d + i) =
                                f32x4{o[t][d][i], o[t][d][i + 1], o[t][d][i + 2], o[t][d][i + 3]} * f;
            } else {
#pragma unroll
                for (int d = 0; d < N; ++d) {
                    i32x4 w;
#pragma unroll
                    for (int i = 0; i < 16; i += 4)
                        w[i / 4] = (int)pack_bytes(
                            requant_bits(o[t][d][i], f), requant_bits(o[t][d][i + 1], f),
                            requant_bits(o[t][d][i + 2], f), requant_bits(o[t][d][i + 3], f));
                    const int32_t c = 16 * N * h2 + 16 * d;
                    if (c < a.hd)
                        *reinterpret_cast<i32x4 *>(reinterpret_cast<int8_t *>(a.y) +
                                                   at(tok, head * a.hd + c, a.n_heads * a.hd, a.y_cb)) = w;
                }
            }
        }
    }
}

// tq: queries of a workgroup
template <int N, int QT, int NW, int SPLIT, bool LISTS>
sl_status launch_shape(AttnArgs &a, int32_t tq, int32_t max_len, hipStream_t s)
{
    a.tq = tq;
    a.tiles = (max_len + tq - 1) / tq;
    a.n_items = (int64_t)a.tiles * a.n_heads * a.n_seq;
    if (a.n_items > 0x7fffffff / (64 * NW * SPLIT)) {
        set_error("too many work items for one launch");
        return SL_ERR_UNSUPPORTED;
    }
    hipLaunchKernelGGL((attention_kernel<N, QT, NW, SPLIT, LISTS>), dim3((uint32_t)a.n_items),
                       dim3(64 * NW * SPLIT), 0, s, a);
    HIP_TRY(hipGetLastError());
    // (formatted once: this is on the path of every call)
    static const std::string name = "attention " + std::to_string(32 * N) + "," + std::to_string(QT) + "," +
                                    std::to_string(NW) + "," + std::to_string(SPLIT) + (LISTS ? " lists" : "");
    set_last_path("%s", name.c_str());
    return SL_OK;
}

template <int N>
sl_status launch_head(AttnArgs &a, const sl_attention_args &args, hipStream_t s)
{
    const int32_t n = args.max_len, qb = args.query_block, tq = args.blocks ? std::min(qb, 32) : 32;
    const int64_t heads = (int64_t)args.n_heads * args.n_seq;
    a.halvings = 0;
    // Keys split over the waves, where 32 queries a workgroup (16 with query_block 16) make no more workgroups than the
    // CUs hold at once: two each, one of heads over 64 features; four in long sequences of heads to 32. Dense: 384 tokens
    // of 12 heads 8.6 us against 10.7, 1024 of 16 heads 17.7 against 21.7, 4096 of 4 heads 46 against 68; 2048 of 12
    // heads (768 workgroups) 39 against 38, 1024 of 24 heads 26 against 22, and 128 tokens (two chunks) 7.0 against 6.5.
    // Heads of 32 features: 1024 tokens of 32 heads (1024 workgroups) 18 against 21, 256 of 128 heads 11.0 against 9.1.
    // Heads of 128: 4096 tokens of 2 heads (256 workgroups) 50 against 107, 1024 of 12 heads 37 against 34. Lists at 4096
    // tokens of 4 heads (512 workgroups) with query_block 64: 16 blocks 18 against 26, 4 blocks 10.2 against 11.1; of 8
    // heads with 128: 16 blocks 32 against 24.
    const int64_t groups = heads * ((n + tq - 1) / tq);
    const int64_t most = N > 2 ? 256 : N == 1 && !args.blocks && n >= 1024 ? 1024 : 512;
    if (groups <= most && (args.blocks ? args.top_k >= 4 : n >= 256)) {
        if (!args.blocks) return launch_shape<N, 1, 1, 4, false>(a, 32, n, s);
        a.halvings = __builtin_ctz(qb / tq);
        return launch_shape<N, 1, 1, 4, true>(a, tq, n, s);
    }
    if (!args.blocks) {
        // Two tiles a wave stage and read a chunk half as often, where 256-query items still fill the CUs twice and the
        // last one of a sequence is a small part: 8192 tokens of 16 heads 365 us against 393, 8 x 2048 of 12 heads 148
        // against 155; 4096 tokens of 12 heads (192 items) 87 against 80.
        if constexpr (N <= 2)
            if (n >= 1024 && heads * ((n + 255) / 256) >= 512) return launch_shape<N, 2, 4, 1, false>(a, 256, n, s);
        return launch_shape<N, 1, 4, 1, false>(a, 128, n, s);
    }
    // As many waves as have queries, against four, 16 blocks at 8192 tokens of 12 heads with query_block 64, 32 and 16:
    // of 64 features 51, 73 and 138 us against 63, 86 and 173, of 96 features 83, 105 and 200 against 103, 163 and 322.
    // (One or two waves would hold the chunk of a head of 128 in too many registers: 8 heads at 4096 tokens with
    // query_block 32 90 against 66.)
    if constexpr (N <= 3) {
        if (qb <= 32) return launch_shape<N, 1, 1, 1, true>(a, qb, n, s);
        if (qb == 64) return launch_shape<N, 1, 2, 1, true>(a, qb, n, s);
    }
    return launch_shape<N, 1, 4, 1, true>(a, qb, n, s);
}

// --- choice of key blocks ----------------------------------------------------

struct SelectArgs {
    const int8_t *x;
    const int32_t *seq_start, *key_len;
    int16_t *pooled;  // [n_kv][head_dim / 8][slots][8]
    int32_t *blocks;
    int64_t m, slots;
    int32_t n_seq, n_heads, n_kv, hd, cols, x_cb, top_k, qb, n_qb, max_blocks;
    int32_t seq0, head0;  // first of this launch
};

// Pooled keys: one wave a key block and 64 features of the keys, 4 features a
// lane, and every 4th key; all 16 loads of a lane are in flight together (16384
// tokens of 12 heads of 64: 5.1 us, 2.5 TB/s).
__global__ __launch_bounds__(256) void pool_keys_kernel(const SelectArgs a)
{
    const int32_t seq = a.seq0 + blockIdx.z, b = blockIdx.y, lane = threadIdx.x & 63;
    const Span sp = span_of(a.seq_start, a.key_len, seq, a.m);
    const int32_t have = min(sp.keys - b * kChunk, kChunk);
    const int32_t c = (blockIdx.x * 4 + threadIdx.x / 64) * 64 + lane % 16 * 4;  // of the key columns
    if (have <= 0) return;
    const bool mine = c < a.n_kv * a.hd;
    const Rows rows(a.x, sp.first + b * kChunk, a.cols, a.x_cb);
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const int32_t key = 4 * j + lane / 16;
        w[j] = 0;
        if (mine && key < have)
            w[j] = *reinterpret_cast<const uint32_t *>(rows.base + rows.offset(key, a.n_heads * a.hd + c));
    }
    int32_t sum[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 16; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = __builtin_amdgcn_sdot4((int)w[j], 1 << (8 * i), sum[i], false);
    i16x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        sum[i] += __shfl_xor(sum[i], 16);
        sum[i] += __shfl_xor(sum[i], 32);
        // (64 sum / have is a half-integer or further than 1 / 128 from one, so its fp32 value rounds as it does)
        out[i] = have == kChunk ? (int16_t)sum[i] : (int16_t)__builtin_rintf((float)(sum[i] * kChunk) / (float)have);
    }
    const int64_t slot = sp.first / kChunk + seq + b;
    if (mine && lane < 16)
        *reinterpret_cast<i16x4 *>(a.pooled + ((int64_t)(c / 8) * a.slots + slot) * 8 + c % 8) = out;
}

// One wave a head and query block: the sum of its queries, the scores of a
// lane's VPL key blocks, and the top_k largest. A score has up to 36 bits:
// products are summed 8 at a time in 32 bits (8 * 2^14 * 2^13 < 2^31), then in
// 64. The top_k-th largest is found bit by bit, by counting. (Bound by the
// latency of its steps: four query blocks a wave, which read the pooled keys a
// quarter as often, took 29 us against 17 at 16384 tokens; now 13.8.)
template <int VPL>
__global__ __launch_bounds__(64) void select_blocks_kernel(const SelectArgs a)
{
    __shared__ int32_t qsum[128];
    __shared__ __attribute__((aligned(16))) int16_t q16[128];
    const int lane = threadIdx.x;
    const int32_t qb = blockIdx.x, head = a.head0 + blockIdx.y, seq = a.seq0 + blockIdx.z;
    const Span sp = span_of(a.seq_start, a.key_len, seq, a.m);
    int32_t *list = a.blocks + (((int64_t)seq * a.n_heads + head) * a.n_qb + qb) * a.top_k;
    const int32_t rows_n = min(sp.n - qb * a.qb, a.qb);
    const int32_t nb = rows_n > 0 ? min((sp.keys + kChunk - 1) / kChunk, a.max_blocks) : 0;
    const int32_t take = min(nb, a.top_k);
    if (nb <= a.top_k) {  // nothing to choose
        for (int32_t i = lane; i < a.top_k; i += 64) list[i] = i < take ? i : -1;
        return;
    }
    qsum[lane] = qsum[lane + 64] = 0;
    __syncthreads();
    {
        // 4 features a lane; lanes beyond the head's features take other rows
        const int quads = a.hd / 4, d = lane % quads * 4, r0 = lane / quads, per = 64 / quads;
        if (r0 < per) {
            int32_t sum[4] = {0, 0, 0, 0};
            const Rows rows(a.x, sp.first + qb * a.qb, a.cols, a.x_cb);
#pragma unroll 8
            for (int32_t r = r0; r < rows_n; r += per) {
                const int32_t w = *reinterpret_cast<const int32_t *>(rows.base + rows.offset(r, head * a.hd + d));
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j] = __builtin_amdgcn_sdot4(w, 1 << (8 * j), sum[j], false);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) atomicAdd(&qsum[d + j], sum[j]);  // (whole numbers: the order does not matter)
        }
    }
    __syncthreads();
    q16[lane] = (int16_t)qsum[lane];
    q16[lane + 64] = (int16_t)qsum[lane + 64];
    __syncthreads();
    const int32_t kv = head / (a.n_heads / a.n_kv);
    const int16_t *pooled = a.pooled + ((int64_t)kv * (a.hd / 8) * a.slots + sp.first / kChunk + seq) * 8;
    int64_t v[VPL];
    constexpr int G = std::min(VPL, 4);  // blocks whose loads are in flight together
#pragma unroll
    for (int j0 = 0; j0 < VPL; j0 += G) {
#pragma unroll
        for (int j = 0; j < G; ++j)
            v[j0 + j] = (j0 + j) * 64 + lane < nb ? (int64_t)1 << 36 : -1;  // (-1: no such block)
#pragma unroll 4
        for (int d8 = 0; d8 < a.hd / 8; ++d8) {
            const i16x8 q = *reinterpret_cast<const i16x8 *>(&q16[8 * d8]);
            i16x8 k[G];
#pragma unroll
            for (int j = 0; j < G; ++j) {
                k[j] = i16x8{0, 0, 0, 0, 0, 0, 0, 0};
                if ((j0 + j) * 64 + lane < nb)
                    k[j] = *reinterpret_cast<const i16x8 *>(pooled + (d8 * a.slots + (j0 + j) * 64 + lane) * 8);
            }
#pragma unroll
            for (int j = 0; j < G; ++j) {
                int32_t s = 0;
#pragma unroll
                for (int e = 0; e < 8; e += 2)
                    s = __builtin_amdgcn_sdot2(i16x2{k[j][e], k[j][e + 1]}, i16x2{q[e], q[e + 1]}, s, false);
                v[j0 + j] += s;
            }
        }
    }
    // the largest t that top_k values or more reach
    int64_t t = 0;
    for (int bit = 36; bit >= 0; --bit) {
        const int64_t want = t | ((int64_t)1 << bit);
        int32_t count = 0;
#pragma unroll
        for (int j = 0; j < VPL; ++j) count += __popcll(__ballot(v[j] >= want));
        if (count >= take) t = want;
    }
    int32_t over = 0;
#pragma unroll
    for (int j = 0; j < VPL; ++j) over += __popcll(__ballot(v[j] > t));
    int32_t ties = take - over, out = 0;  // of those that equal t, the first `ties`
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const uint64_t eq = __ballot(v[j] == t);
        const bool chosen = v[j] > t || (v[j] == t && __popcll(eq & below) < ties);
        ties -= min(ties, (int32_t)__popcll(eq));
        const uint64_t sel = __ballot(chosen);
        if (chosen) list[out + __popcll(sel & below)] = j * 64 + lane;
        out += __popcll(sel);
    }
}

}  // namespace

sl_status launch_attention(const sl_attention_args &args, void *stream)
{
    AttnArgs a{};
    a.x = args.x;
    a.seq_start = args.seq_start;
    a.key_len = args.key_len;
    a.blocks = args.blocks;
    a.y = args.y;
    a.m = args.m_tokens;
    a.n_seq = args.n_seq;
    a.n_heads = args.n_heads;
    a.n_kv = args.n_kv_heads;
    a.hd = args.head_dim;
    a.cols = (args.n_heads + 2 * args.n_kv_heads) * args.head_dim;
    a.x_cb = args.x_layout == SL_LAYOUT_T16X32 ? (a.cols + 31) / 32 : 0;
    a.y_cb = args.y_layout == SL_LAYOUT_T16X32 ? (a.n_heads * a.hd + 31) / 32 : 0;
    if (args.blocks) {
        a.top_k = args.top_k;
        a.n_qb = (args.max_len + args.query_block - 1) / args.query_block;
    }
    const Exponent e = exponent_of((double)args.x_scale * args.x_scale * args.softmax_scale);
    a.c2 = e.c2;
    a.k2 = e.k2;
    a.xs = args.x_scale;
    a.y_f32 = args.kind == SL_EPI_F32;
    a.inv_so = args.kind == SL_EPI_I8 ? 1.0f / args.out_scale : 1.0f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch ((a.hd + 31) / 32) {
    case 1: return launch_head<1>(a, args, s);
    case 2: return launch_head<2>(a, args, s);
    case 3: return launch_head<3>(a, args, s);
    default: return launch_head<4>(a, args, s);
    }
}

sl_status launch_attention_select(const sl_attention_args &args, int32_t *blocks, void *workspace, void *stream)
{
    SelectArgs a{};
    a.x = args.x;
    a.seq_start = args.seq_start;
    a.key_len = args.key_len;
    a.pooled = static_cast<int16_t *>(workspace);
    a.blocks = blocks;
    a.m = args.m_tokens;
    a.slots = pooled_slots(args);
    a.n_seq = args.n_seq;
    a.n_heads = args.n_heads;
    a.n_kv = args.n_kv_heads;
    a.hd = args.head_dim;
    a.cols = (args.n_heads + 2 * args.n_kv_heads) * args.head_dim;
    a.x_cb = args.x_layout == SL_LAYOUT_T16X32 ? (a.cols + 31) / 32 : 0;
    a.top_k = args.top_k;
    a.qb = args.query_block;
    a.n_qb = (args.max_len + a.qb - 1) / a.qb;
    a.max_blocks = (args.max_len + kChunk - 1) / kChunk;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    constexpr int32_t kMostGrid = 65535;  // workgroups of a launch in its second and third dimension
    for (int64_t s0 = 0; s0 < a.n_seq; s0 += kMostGrid) {
        a.seq0 = (int32_t)s0;
        const int32_t seqs = std::min(a.n_seq - a.seq0, kMostGrid);
        hipLaunchKernelGGL(pool_keys_kernel, dim3((a.n_kv * a.hd + 255) / 256, a.max_blocks, seqs), dim3(256), 0, s, a);
        HIP_TRY(hipGetLastError());
        for (int32_t h0 = 0; h0 < a.n_heads; h0 += kMostGrid) {
            a.head0 = h0;
            const dim3 grid(a.n_qb, std::min(a.n_heads - h0, kMostGrid), seqs);
            if (a.max_blocks <= 64)
                hipLaunchKernelGGL(select_blocks_kernel<1>, grid, dim3(64), 0, s, a);
            else if (a.max_blocks <= 256)
                hipLaunchKernelGGL(select_blocks_kernel<4>, grid, dim3(64), 0, s, a);
            else if (a.max_blocks <= 1024)
                hipLaunchKernelGGL(select_blocks_kernel<16>, grid, dim3(64), 0, s, a);
            else
                hipLaunchKernelGGL(select_blocks_kernel<64>, grid, dim3(64), 0, s, a);
            HIP_TRY(hipGetLastError());
        }
    }
    return SL_OK;
}

}  // namespace sl
