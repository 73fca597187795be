// attention_run and attention_select (gfx950).
//
// Attention. For one head and a tile of queries, over chunks of 64 keys:
//   S = K Q^T            int8 x int8 -> int32 on v_mfma_i32_16x16x64_i8, exact
//   P = 2^(c (S - m))    m: running maximum of a query's S
//   l += sum P, O += V^T P^T   on v_mfma_f32_16x16x32_f16
// and y = x_scale O / l. S is computed transposed (keys are the matrix
// instruction's rows, queries its columns) so that a lane's scores all belong
// to one query and lie where the second product takes its right operand from:
// lane group g of a 16-key tile holds keys 4g .. 4g+3, and a pair of tiles'
// scores, rounded to 16 bits, are the 8 values a lane gives to a 32-key
// product. That product may take the keys in any order as long as V's operand
// has them in the same one, so V is laid out in LDS in that order.
//
// The integer scores meet the exponential without a conversion: the
// accumulators start at the bits of 1.5 * 2^23 as a float, less m, so that the
// finished sums read as floats are 1.5 * 2^23 + (S - m) exactly
// (|S - m| < 2^22 for heads of up to 128 features), and one fused multiply-add
// gives the exponent.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "encoder.h"
#include "sl_device.h"

namespace sl {

namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kChunk = SL_KEY_BLOCK;      // keys of a step
constexpr int32_t kMagic = 0x4B400000;    // bits of 1.5 * 2^23
constexpr float kMagicF = 12582912.0f;
// P carries a factor 2^kBias: values down to 2^-21 of the largest stay normal 16-bit floats
constexpr float kBias = 7.0f;
// m may lag behind the running maximum by 2^kLag (P <= 2^(kBias + 1 + kLag) < 65504)
constexpr float kLag = 7.0f;

struct AttnArgs {
    const int8_t *x;
    const int32_t *seq_start, *key_len, *blocks;
    void *y;
    int64_t m;
    int64_t n_items;
    int32_t n_seq, tiles, n_heads, n_kv, hd, cols, x_cb, y_cb;
    int32_t top_k, n_qb;
    float c2, k2, inv_so, xs;
    int32_t lag;
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

// byte offset of feature c of token t
__device__ __forceinline__ int64_t at(int64_t t, int32_t c, int32_t cols, int32_t cb)
{
    return cb ? t16x32_offset(t, c, cb) : t * cols + c;
}

__device__ __forceinline__ int group_max(int v)
{
    v = max(v, __shfl_xor(v, 16));
    return max(v, __shfl_xor(v, 32));
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

// DT: 16-feature tiles of a head (head_dim <= 16 DT); QT: 16-query tiles of a
// wave; NW: waves of a workgroup.
template <int DT, int QT, int NW, bool F32, bool LISTS>
__global__ __launch_bounds__(64 * NW) void attention_kernel(const AttnArgs a)
{
    constexpr int D = 16 * DT;
    constexpr int KK = (D + 63) / 64;          // 64-feature products of a score
    constexpr int KS = D + 16, VS = 2 * kChunk + 16;  // LDS bytes of a key, and of a feature of V
    constexpr int TQ = 16 * QT * NW;
    __shared__ __attribute__((aligned(16))) char ks[kChunk * KS];
    __shared__ __attribute__((aligned(16))) char vs[D * VS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, n16 = lane & 15;
    const int64_t item = xcd_work_index(blockIdx.x, a.n_items);
    const int32_t tile = (int32_t)(item % a.tiles);
    const int32_t head = (int32_t)(item / a.tiles % a.n_heads);
    const int32_t seq = (int32_t)(item / a.tiles / a.n_heads);
    const Span sp = span_of(a.seq_start, a.key_len, seq, a.m);
    const int32_t kv = head / (a.n_heads / a.n_kv);
    const int32_t kcol = (a.n_heads + kv) * a.hd, vcol = (a.n_heads + a.n_kv + kv) * a.hd;
    const int32_t n_blocks = (sp.keys + kChunk - 1) / kChunk;

    for (int32_t qt = tile; (int64_t)qt * TQ < sp.n; qt += a.tiles) {
        const int32_t q0 = qt * TQ + wave * 16 * QT;
        i32x4 q[QT][KK];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int h = 0; h < KK; ++h) {
                const int32_t qi = q0 + 16 * t + n16, d = 64 * h + 16 * g;
                q[t][h] = i32x4{0, 0, 0, 0};
                if (qi < sp.n && d < a.hd)
                    q[t][h] = *reinterpret_cast<const i32x4 *>(
                        a.x + at((int64_t)sp.first + qi, head * a.hd + d, a.cols, a.x_cb));
            }
        }
        f32x4 o[QT][DT], l[QT];
        int32_t m[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            m[t] = 0;
            l[t] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int d = 0; d < DT; ++d) o[t][d] = f32x4{0, 0, 0, 0};
        }
        const int32_t steps = LISTS ? (qt < a.n_qb ? a.top_k : 0) : n_blocks;
        const int32_t *list = a.blocks + (((int64_t)seq * a.n_heads + head) * a.n_qb + qt) * a.top_k;
        bool first = true;
        for (int32_t step = 0; step < steps; ++step) {
            const int32_t b = LISTS ? list[step] : step;
            if (LISTS && (uint32_t)b >= (uint32_t)n_blocks) continue;
            const int32_t k0 = b * kChunk, have = min(sp.keys - k0, kChunk);
            __syncthreads();
            // stage: keys as they are (16-byte pieces), values by 4 keys x 4 features
            for (int i = tid; i < kChunk * DT; i += 64 * NW) {
                const int key = i / DT, d = i % DT * 16;
                i32x4 v = {0, 0, 0, 0};
                if (key < have && d < a.hd)
                    v = *reinterpret_cast<const i32x4 *>(
                        a.x + at((int64_t)sp.first + k0 + key, kcol + d, a.cols, a.x_cb));
                *reinterpret_cast<i32x4 *>(ks + key * KS + d) = v;
            }
            for (int i = tid; i < kChunk / 4 * D / 4; i += 64 * NW) {
                const int kq = i / (D / 4), d = i % (D / 4) * 4;  // keys 4 kq .. 4 kq + 3
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (4 * kq + j < have && d < a.hd)
                        w[j] = *reinterpret_cast<const uint32_t *>(
                            a.x + at((int64_t)sp.first + k0 + 4 * kq + j, vcol + d, a.cols, a.x_cb));
                }
                u32x2 out[4];
                transpose_to_f16(w, out);
                // place of the 4 keys in a feature's row: their lane group's 8 of the 32, first or second tile
                const int pos = (kq >> 3) * 32 + (kq & 3) * 8 + ((kq >> 2) & 1) * 4;
                // row of feature 4 DT x + 4 y + j: 16 y + 4 x + j, so that a lane's sums are consecutive features
                const int row = 16 * ((d >> 2) % DT) + 4 * (d / (4 * DT));
#pragma unroll
                for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x2 *>(vs + (row + j) * VS + 2 * pos) = out[j];
            }
            __syncthreads();
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                i32x4 s[4];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) {
                    const int32_t z = kMagic - m[t];
                    s[kt] = i32x4{z, z, z, z};
#pragma unroll
                    for (int h = 0; h < KK; ++h) {
                        i32x4 k = {0, 0, 0, 0};
                        if (64 * h + 16 * g < D)
                            k = *reinterpret_cast<const i32x4 *>(ks + (16 * kt + n16) * KS + 64 * h + 16 * g);
                        s[kt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(k, q[t][h], s[kt], 0, 0, 0);
                    }
                }
                if (have < kChunk) {
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (16 * kt + 4 * g + r >= have) s[kt][r] = 0;
                }
                int top = s[0][0];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) top = max(top, s[kt][r]);
                const int up = group_max(top) - kMagic;
                if (first || __any(up > a.lag)) {
                    const int by = first ? up : max(up, 0);
                    const float f = first ? 1.0f : __builtin_amdgcn_exp2f(-(float)by * a.c2);
                    m[t] += by;
                    l[t] *= f;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[t][d] *= f;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[kt][r] -= by;
                }
                f16x8 p[2], p2[2];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) {
                    float e[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        e[r] = __builtin_amdgcn_exp2f(fmaf(__int_as_float(s[kt][r]), a.c2, a.k2));
                        if (have < kChunk && 16 * kt + 4 * g + r >= have) e[r] = 0.0f;
                    }
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        const auto hi = __builtin_amdgcn_cvt_pkrtz(e[r], e[r + 1]);
                        p[kt / 2][(kt & 1) * 4 + r] = hi[0];
                        p[kt / 2][(kt & 1) * 4 + r + 1] = hi[1];
                        if constexpr (F32) {
                            const auto lo = __builtin_amdgcn_cvt_pkrtz(e[r] - (float)hi[0], e[r + 1] - (float)hi[1]);
                            p2[kt / 2][(kt & 1) * 4 + r] = lo[0];
                            p2[kt / 2][(kt & 1) * 4 + r + 1] = lo[1];
                        }
                    }
                }
                const _Float16 one = (_Float16)1.0f;
                const f16x8 ones = {one, one, one, one, one, one, one, one};
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    l[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[w], l[t], 0, 0, 0);
                    if constexpr (F32) l[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p2[w], l[t], 0, 0, 0);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const f16x8 v =
                            *reinterpret_cast<const f16x8 *>(vs + (16 * d + n16) * VS + 64 * w + 16 * g);
                        o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[w], o[t][d], 0, 0, 0);
                        if constexpr (F32) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p2[w], o[t][d], 0, 0, 0);
                    }
                }
            }
            first = false;
        }
        // lane group g holds features 4 DT g .. 4 DT g + 4 DT - 1 of its query
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int32_t qi = q0 + 16 * t + n16;
            if (qi >= sp.n) continue;
            const int64_t tok = (int64_t)sp.first + qi;
            const float f = first ? 0.0f : a.xs / l[t][0];
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int32_t c = 4 * DT * g + 4 * d;
                if (c >= a.hd) continue;
                const f32x4 v = o[t][d] * f;
                if constexpr (F32) {
                    store_nt(reinterpret_cast<float *>(a.y) + tok * (a.n_heads * a.hd) + head * a.hd + c, v);
                } else {
                    *reinterpret_cast<uint32_t *>(reinterpret_cast<int8_t *>(a.y) +
                                                  at(tok, head * a.hd + c, a.n_heads * a.hd, a.y_cb)) =
                        pack_bytes(requant_bits(v[0], a.inv_so), requant_bits(v[1], a.inv_so),
                                   requant_bits(v[2], a.inv_so), requant_bits(v[3], a.inv_so));
                }
            }
        }
    }
}

template <int DT, int QT, int NW, bool LISTS>
sl_status launch_kind(AttnArgs &a, int32_t kind, int32_t max_len, hipStream_t s)
{
    constexpr int TQ = 16 * QT * NW;
    a.tiles = (max_len + TQ - 1) / TQ;
    a.n_items = (int64_t)a.tiles * a.n_heads * a.n_seq;
    if (a.n_items > 0x7fffffff / (64 * NW)) {
        set_error("too many work items for one launch");
        return SL_ERR_UNSUPPORTED;
    }
    if (kind == SL_EPI_F32)
        hipLaunchKernelGGL((attention_kernel<DT, QT, NW, true, LISTS>), dim3((uint32_t)a.n_items), dim3(64 * NW), 0, s,
                           a);
    else
        hipLaunchKernelGGL((attention_kernel<DT, QT, NW, false, LISTS>), dim3((uint32_t)a.n_items), dim3(64 * NW), 0,
                           s, a);
    HIP_TRY(hipGetLastError());
    return SL_OK;
}

template <int DT>
sl_status launch_head(AttnArgs &a, const sl_attention_args &args, hipStream_t s)
{
    if (!args.blocks) return launch_kind<DT, 1, 4, false>(a, args.kind, args.max_len, s);
    switch (args.query_block) {
    case 16: return launch_kind<DT, 1, 1, true>(a, args.kind, args.max_len, s);
    case 32: return launch_kind<DT, 1, 2, true>(a, args.kind, args.max_len, s);
    case 64: return launch_kind<DT, 1, 4, true>(a, args.kind, args.max_len, s);
    default: return launch_kind<DT, 2, 4, true>(a, args.kind, args.max_len, s);
    }
}

// --- choice of key blocks ----------------------------------------------------

struct SelectArgs {
    const int8_t *x;
    const int32_t *seq_start, *key_len;
    int16_t *pooled;  // [n_kv][head_dim / 8][slots][8]
    int32_t *blocks;
    int64_t m, slots;
    int32_t n_seq, n_heads, n_kv, hd, cols, x_cb, top_k, qb, n_qb, max_blocks;
};

// Pooled keys: one thread a key block and 4 features, over the block's keys.
__global__ __launch_bounds__(256) void pool_keys_kernel(const SelectArgs a)
{
    const int32_t seq = blockIdx.z, b = blockIdx.y;
    const Span sp = span_of(a.seq_start, a.key_len, seq, a.m);
    const int32_t have = min(sp.keys - b * kChunk, kChunk);
    const int32_t c = (blockIdx.x * 256 + threadIdx.x) * 4;  // of the key columns
    if (have <= 0 || c >= a.n_kv * a.hd) return;
    int32_t sum[4] = {0, 0, 0, 0};
    for (int32_t j = 0; j < have; ++j) {
        const int32_t w = *reinterpret_cast<const int32_t *>(
            a.x + at((int64_t)sp.first + b * kChunk + j, a.n_heads * a.hd + c, a.cols, a.x_cb));
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += (int8_t)(w >> (8 * i));
    }
    const int64_t slot = sp.first / kChunk + seq + b;
    int16_t *out = a.pooled + ((int64_t)(c / 8) * a.slots + slot) * 8 + c % 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (64 sum / have is a half-integer or further than 1 / 128 from one, so its fp32 value rounds as it does)
        out[i] = have == kChunk ? (int16_t)sum[i] : (int16_t)__builtin_rintf((float)(sum[i] * kChunk) / (float)have);
    }
}

// One wave a query block and head: the sum of its queries, a score a key block
// (VPL a lane), and the top_k of them. A score has up to 36 bits: products are
// summed 8 at a time in 32 bits (8 * 2^14 * 2^13 < 2^31), then in 64. The
// top_k-th largest is found bit by bit, by counting.
template <int VPL>
__global__ __launch_bounds__(64) void select_blocks_kernel(const SelectArgs a)
{
    __shared__ int32_t qsum[128];
    const int lane = threadIdx.x;
    const int32_t qb = blockIdx.x, head = blockIdx.y, seq = blockIdx.z;
    const Span sp = span_of(a.seq_start, a.key_len, seq, a.m);
    int32_t *list = a.blocks + (((int64_t)seq * a.n_heads + head) * a.n_qb + qb) * a.top_k;
    const int32_t rows = min(sp.n - qb * a.qb, a.qb);
    const int32_t nb = rows > 0 ? min((sp.keys + kChunk - 1) / kChunk, a.max_blocks) : 0;
    const int32_t take = min(nb, a.top_k);
    for (int32_t i = take + lane; i < a.top_k; i += 64) list[i] = -1;
    if (nb == 0) return;
    if (nb <= a.top_k) {
        for (int32_t i = lane; i < nb; i += 64) list[i] = i;
        return;
    }
    for (int d = lane * 4; d < 128; d += 256) {
#pragma unroll
        for (int i = 0; i < 4; ++i) qsum[d + i] = 0;
    }
    __syncthreads();
    {
        // 4 features a lane; lanes beyond the head's features take other rows
        const int quads = a.hd / 4, d = lane % quads * 4, r0 = lane / quads, per = 64 / quads;
        int32_t sum[4] = {0, 0, 0, 0};
        if (r0 < per) {
            for (int32_t r = r0; r < rows; r += per) {
                const int32_t w = *reinterpret_cast<const int32_t *>(
                    a.x + at((int64_t)sp.first + (int64_t)qb * a.qb + r, head * a.hd + d, a.cols, a.x_cb));
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += (int8_t)(w >> (8 * i));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) atomicAdd(&qsum[d + i], sum[i]);  // (whole numbers: the order does not matter)
        }
    }
    __syncthreads();
    const int32_t kv = head / (a.n_heads / a.n_kv);
    const int64_t slot = sp.first / kChunk + seq;
    const int16_t *pooled = a.pooled + (int64_t)kv * (a.hd / 8) * a.slots * 8;
    int64_t v[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int32_t b = i * 64 + lane;
        v[i] = -1;  // below every score's unsigned form
        if (b < nb) {
            int64_t score = (int64_t)1 << 36;
            for (int d8 = 0; d8 < a.hd / 8; ++d8) {
                const int16_t *k = pooled + ((int64_t)d8 * a.slots + slot + b) * 8;
                int32_t s = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) s += qsum[d8 * 8 + j] * (int32_t)k[j];
                score += s;
            }
            v[i] = score;
        }
    }
    // the largest t that take values or more reach
    int64_t t = 0;
    for (int bit = 36; bit >= 0; --bit) {
        const int64_t want = t | ((int64_t)1 << bit);
        int32_t count = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) count += __popcll(__ballot(v[i] >= want));
        if (count >= take) t = want;
    }
    int32_t over = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) over += __popcll(__ballot(v[i] > t));
    int32_t ties = take - over, out = 0;  // of those that equal t, the first `ties`
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const uint64_t eq = __ballot(v[i] == t);
        const bool chosen = v[i] > t || (v[i] == t && __popcll(eq & below) < ties);
        ties -= min(ties, (int32_t)__popcll(eq));
        const uint64_t sel = __ballot(chosen);
        if (chosen) list[out + __popcll(sel & below)] = i * 64 + lane;
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
    // log2 units a whole number of S is worth, rounded to 22 bits: times 1.5 * 2^23 it is then a float itself,
    // and the exponent of P loses nothing to that offset
    const double c2 = (double)args.x_scale * args.x_scale * args.softmax_scale * 1.4426950408889634;
    int e = 0;
    const double frac = frexp(c2, &e);
    a.c2 = (float)ldexp(nearbyint(ldexp(frac, 22)), e - 22);
    a.k2 = kBias - kMagicF * a.c2;
    a.lag = (int32_t)std::min<double>(kLag / std::max((double)a.c2, 1e-30), 1 << 23);
    a.xs = args.x_scale;
    a.inv_so = args.kind == SL_EPI_I8 ? 1.0f / args.out_scale : 1.0f;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.hd <= 32) return launch_head<2>(a, args, s);
    if (a.hd <= 64) return launch_head<4>(a, args, s);
    return launch_head<8>(a, args, s);
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
    if (a.n_seq > 65535 || a.n_heads > 65535) {
        set_error("more than 65535 sequences or heads");
        return SL_ERR_UNSUPPORTED;
    }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(pool_keys_kernel, dim3((a.n_kv * a.hd / 4 + 255) / 256, a.max_blocks, a.n_seq), dim3(256), 0, s,
                       a);
    HIP_TRY(hipGetLastError());
    const dim3 grid(a.n_qb, a.n_heads, a.n_seq);
    if (a.max_blocks <= 256)
        hipLaunchKernelGGL(select_blocks_kernel<4>, grid, dim3(64), 0, s, a);
    else if (a.max_blocks <= 1024)
        hipLaunchKernelGGL(select_blocks_kernel<16>, grid, dim3(64), 0, s, a);
    else
        hipLaunchKernelGGL(select_blocks_kernel<64>, grid, dim3(64), 0, s, a);
    HIP_TRY(hipGetLastError());
    return SL_OK;
}

}  // namespace sl
