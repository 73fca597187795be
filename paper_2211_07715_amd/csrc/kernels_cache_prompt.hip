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
//             one with a page that is none) and those that move m a step at a time.
#include <hip/hip_runtime.h>

#include "cache_device.h"

namespace sl {

namespace {

typedef const __attribute__((address_space(4))) int32_t *ScalarTable;  // read through the scalar cache

// N: 32-feature tiles of a head; QT: tiles of 32 queries a wave
template <int N, int QT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(N <= 2 && QT == 1 ? 3 : 2)))
void cache_prompt_kernel(const CacheArgs a)
{
    constexpr int D = 32 * N, PR = N <= 2 ? 2 * N : 8;  // 16-byte pieces of a key's row in LDS
    constexpr int KS = 16 * PR, VS = 2 * kChunk, KB = kChunk * KS, BUF = KB + D * VS;
    constexpr int KP = (16 * PR + 63) / 64, VP = (D + 63) / 64;  // a lane's pieces of 16 tokens' keys and values
    constexpr int KN = N == 3 ? 4 : N;  // whose swap a key's row takes
    constexpr int TQ = 128 * QT;
    __shared__ __attribute__((aligned(16))) char lds[2 * BUF];
    const int lane = threadIdx.x & 63, half = lane >> 5, n32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // tiles of a sequence from the last, which sees the most keys, for all heads and sequences
    const uint32_t pairs = (uint32_t)a.n_kv * (uint32_t)a.n_seq, pair = blockIdx.x % pairs;
    const int32_t tile0 = a.tiles - 1 - (int32_t)(blockIdx.x / pairs);
    const int32_t kv = (int32_t)(pair % (uint32_t)a.n_kv), seq = (int32_t)(pair / (uint32_t)a.n_kv);
    const Tokens tk = tokens_of(a.seq_start, seq, a.m);
    const int64_t rows = (int64_t)tk.n * a.group;
    const int32_t len = max(a.kv_len[seq], 0);
    const int32_t cached = (int32_t)min((int64_t)len, (int64_t)a.max_pages << a.shift);
    const ScalarTable table = (ScalarTable)(uintptr_t)(a.page_table + (int64_t)seq * a.max_pages);
    const int64_t head_bytes = (int64_t)a.hd << a.shift, page_bytes = 2 * a.n_kv * head_bytes;
    const int8_t *keys = a.cache + kv * head_bytes, *values = keys + a.n_kv * head_bytes;
    const int32_t in_mask = (1 << a.shift) - 1;

    // A lane's pieces of its wave's 16 tokens: bytes from the first one's, and where they go. Row 8 i + 4 h + b of 16 is
    // key 8 h + 4 i + b, as a lane half h of the scores has them.
    uint32_t koff[KP], voff[VP], vdst[VP];
    bool kmine[KP], vmine[VP];
#pragma unroll
    for (int i = 0; i < KP; ++i) {
        const int p = lane + 64 * i, row = 16 * wave + p / PR;
        const int piece = p % PR ^ kswap<KN>(row), key = (row & 3) | (row & 4) << 1 | (row & 8) >> 1;
        kmine[i] = p < 16 * PR && 16 * piece < a.hd;
        koff[i] = (uint32_t)(key * a.hd + 16 * piece);
    }
#pragma unroll
    for (int i = 0; i < VP; ++i) {
        const int d = lane + 64 * i;
        vmine[i] = d < a.hd;
        voff[i] = (uint32_t)d * 16;
        // (lane half h of the product's rows 8 x + 4 h + b then holds features 16 N h + 16 tile + 4 x + b)
        const int row = 32 * (d / 16 % N) + 8 * (d / 4 % 4) + 4 * (d / (16 * N)) + d % 4;
        vdst[i] = KB + row * VS + ((32 * wave) ^ (16 * vswap(row)));
    }
    i32x4 vreg[VP];
    // pages of a chunk: the wave's own, and which of the four are none
    int32_t own = 0;
    uint32_t none = 0;
    const auto entries = [&](int32_t c) __attribute__((always_inline)) {
        none = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int32_t e = table[min((kChunk * c + 16 * j) >> a.shift, a.max_pages - 1)];
            const bool there = (uint32_t)e < (uint32_t)a.n_pages;
            none |= there ? 0u : 1u << j;
            if (j == wave) own = there ? e : 0;
        }
    };
    const auto load = [&](int32_t c, char *buf) __attribute__((always_inline)) {
        const int64_t from = own * page_bytes + ((kChunk * c + 16 * wave) & in_mask) * (int64_t)a.hd;
        const auto k = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(keys + from), 0, 0x7fffffff, kRsrcWord3);
        const auto v = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(values + from), 0, 0x7fffffff, kRsrcWord3);
#pragma unroll
        for (int i = 0; i < KP; ++i)
            if (kmine[i]) load_to_lds(k, buf + wave * 16 * KS + 1024 * i, koff[i], 0);
#pragma unroll
        for (int i = 0; i < VP; ++i)
            if (vmine[i]) vreg[i] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(v, voff[i], 0, 0));
    };
    const auto stage = [&](char *buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            if (!vmine[i]) continue;
            uint32_t out[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // a code c as an unsigned byte c + 128 under the byte 0x64 is the 16-bit float 1152 + c
                const uint32_t w = (uint32_t)vreg[i][j] ^ 0x80808080u, e = 0x64646464u;
                const f16x2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
                out[2 * j] = __builtin_bit_cast(
                    uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(e, w, 0x04010400u)) - bias);
                out[2 * j + 1] = __builtin_bit_cast(
                    uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(e, w, 0x04030402u)) - bias);
            }
            *reinterpret_cast<i32x4 *>(buf + vdst[i]) = i32x4{(int)out[0], (int)out[1], (int)out[2], (int)out[3]};
            *reinterpret_cast<i32x4 *>(buf + (vdst[i] ^ 16)) = i32x4{(int)out[4], (int)out[5], (int)out[6], (int)out[7]};
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };

    for (int64_t tile = tile0; tile * TQ < rows; tile += a.tiles) {
        const int64_t first_row = tile * TQ, end_row = min(first_row + TQ, rows);
        const int32_t i0 = (int32_t)(first_row / a.group), g0 = (int32_t)(first_row - (int64_t)i0 * a.group);
        // a lane's query of tile t: token, or -1, and head
        const auto query = [&](int t, int32_t &head) {
            const int32_t x = (wave * QT + t) * 32 + here(n32), y = g0 + x, di = (int32_t)((uint32_t)y / (uint32_t)a.group);
            head = kv * a.group + (y - di * a.group);
            return first_row + x < end_row ? i0 + di : -1;
        };
        const auto sees = [&](int32_t i) { return a.causal ? min(len - tk.n + i + 1, cached) : cached; };
        const int32_t most = sees((int32_t)((end_row - 1) / a.group));
        const int32_t n_chunks = (max(most, 0) + kChunk - 1) / kChunk;
        // keys that the wave's first and last query see
        const int64_t w0 = first_row + wave * 32 * QT, w1 = min(w0 + 32 * QT, end_row);
        const int32_t least = w0 < end_row ? sees((int32_t)(w0 / a.group)) : 0;
        const int32_t mine = w0 < end_row ? (max(sees((int32_t)((w1 - 1) / a.group)), 0) + kChunk - 1) / kChunk : 0;

        i32x4 q[QT][N];
        int32_t limit[QT];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            int32_t head;
            const int32_t i = query(t, head);
            limit[t] = i >= 0 ? sees(i) : 0x7fffffff;
#pragma unroll
            for (int h = 0; h < N; ++h) {
                const int32_t d = 32 * h + 16 * here(half);
                q[t][h] = i32x4{0, 0, 0, 0};
                if (i >= 0 && d < a.hd)
                    q[t][h] = *reinterpret_cast<const i32x4 *>(
                        a.q + at((int64_t)tk.first + i, head * a.hd + d, a.q_cols, a.q_cb));
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
        const auto scores = [&](int t, const char *buf, const i32x16 &from, i32x16 (&s)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                s[kt] = from;
#pragma unroll
                for (int h = 0; h < N; ++h) {
                    const int row = 32 * kt + n32;
                    const i32x4 k = *reinterpret_cast<const i32x4 *>(buf + row * KS + 16 * ((2 * h + half) ^ kswap<KN>(n32)));
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
        // keys that the query does not see: minus infinity, as the bits that the scores are
        const auto mask = [&](int t, int32_t c, uint32_t gone, i32x16 (&s)[2]) __attribute__((always_inline)) {
            const int32_t left = limit[t] - kChunk * c - 8 * half;
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

        int32_t c = 0, buf = 0;
        uint32_t gone = 0;  // which of the chunk's pages are none
        if (n_chunks > 0) {
            entries(0);
            gone = none;
            load(0, lds);
            entries(1);
            stage(lds);
        }
        __syncthreads();
        // every chunk: the next one's loads, this one's work, then the next one goes to LDS
        const auto bring = [&]() __attribute__((always_inline)) {
            if (c + 1 < n_chunks) load(c + 1, lds + (buf ^ BUF));
        };
        const auto advance = [&]() __attribute__((always_inline)) {
            buf ^= BUF;
            ++c;
            gone = none;
            if (c < n_chunks) {
                stage(lds + buf);
                entries(c + 1);
            }
            __syncthreads();
        };
        i32x16 sc[2];
        while (c < mine) {
            bring();
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                scores(t, lds + buf, from_z(t), sc);
                mask(t, c, gone, sc);
                raise(t, largest(sc));
                scores(t, lds + buf, from_z(t), sc);
                mask(t, c, gone, sc);
                l[t] += weights(t, sc);
            }
            multiply(lds + buf);
            advance();
            i32x16 from[QT];
#pragma unroll
            for (int t = 0; t < QT; ++t) from[t] = from_z(t);
            while (kChunk * (c + 1) <= least && !gone) {
                bring();
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
                advance();
            }
        }
        while (c < n_chunks) {  // others' chunks
            bring();
            advance();
        }
        // a lane half holds features 16 N half .. 16 N half + 16 N - 1 of its query
        const int32_t cols = a.n_heads * a.hd;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float sum = pair_sum(l[t]);
            const float f = sum > 0.0f ? a.vs / sum * a.inv_so : 0.0f;
            int32_t head;
            const int32_t i = query(t, head);
            if (i < 0) continue;
            const int64_t tok = (int64_t)tk.first + i;
            const int h2 = here(half);
#pragma unroll
            for (int d = 0; d < N; ++d) {
                const int32_t f0 = 16 * N * h2 + 16 * d;
                if (f0 >= a.hd) continue;
                if (a.y_f32) {
                    float *y = static_cast<float *>(a.y) + tok * cols + head * a.hd + f0;
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        *reinterpret_cast<f32x4 *>(y + e) =
                            f32x4{o[t][d][e], o[t][d][e + 1], o[t][d][e + 2], o[t][d][e + 3]} * f;
                } else {
                    i32x4 w;
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        w[e / 4] = (int)pack_bytes(requant_bits(o[t][d][e], f), requant_bits(o[t][d][e + 1], f),
                                                   requant_bits(o[t][d][e + 2], f), requant_bits(o[t][d][e + 3], f));
                    *reinterpret_cast<i32x4 *>(static_cast<int8_t *>(a.y) + at(tok, head * a.hd + f0, cols, a.y_cb)) = w;
                }
            }
        }
    }
}

template <int N, int QT>
sl_status launch_shape(CacheArgs &a, const sl_cache_attention_args &args, hipStream_t s)
{
    const int64_t tiles = ((int64_t)args.max_new * a.group + 128 * QT - 1) / (128 * QT);
    if ((double)a.n_kv * a.n_seq * (double)tiles > 0x7fffffff / 256) {
        set_error("too many work items for one launch");
        return SL_ERR_UNSUPPORTED;
    }
    a.tiles = (int32_t)tiles;
    hipLaunchKernelGGL((cache_prompt_kernel<N, QT>), dim3((uint32_t)(a.n_kv * a.n_seq * a.tiles)), dim3(256), 0, s, a);
    HIP_TRY(hipGetLastError());
    set_last_path("cache prompt %d,%d", 32 * N, QT);
    return SL_OK;
}

}  // namespace

sl_status launch_cache_prompt(CacheArgs a, const sl_cache_attention_args &args, hipStream_t s)
{
    const Exponent e = exponent_of((double)args.q_scale * args.k_scale * args.softmax_scale);
    a.c2 = e.c2;
    a.k2 = e.k2;
    switch ((a.hd + 31) / 32) {
    case 1: return launch_shape<1, 1>(a, args, s);
    case 2: return launch_shape<2, 1>(a, args, s);
    case 3: return launch_shape<3, 1>(a, args, s);
    default: return launch_shape<4, 1>(a, args, s);
    }
}

}  // namespace sl
