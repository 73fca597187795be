// residual_norm: t = post(y), h = residual_scale r + gate t, u = norm(h) and
// its int8 codes, in one pass (gfx950).
//
// Bound by memory: per element it reads y and r (4 or 1 bytes each) and writes
// what the caller keeps, against some 20 vector instructions. So every input is
// read once, a whole row stays in registers between the sums (mean, then the
// squared deviations from it: two passes over registers, not over memory), and
// all of a row's loads are issued before any of them is used.
//
// A row belongs to W waves of one workgroup, each lane holding IT groups of 4
// consecutive features, 256 W apart: fp32 rows move in 16-byte pieces a lane,
// int8 rows in either layout in 4-byte ones. W = 1 (up to 1024 features of many
// rows) needs no barrier and no LDS.
//
// Measured, replayed from a graph: 4096 x 768, fp32 in and int8 out, 8.4 us (4.9
// TB/s, of 5.1 that a copy of 1 GiB reaches); 49152 x 1024, int8 y, norms on both
// sides, h kept, 119 us (4.2 TB/s); 1531 x 1001, fp32, 8.1 us (3.2 TB/s); 128 x 768
// 3.2 us; 49152 x 768, codes to codes, all in pieces of 4 bytes, 40 us (2.8 TB/s).
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "encoder.h"
#include "sl_device.h"

namespace sl {

namespace {

struct NormArgs {
    sl_residual_norm_args a;
    int32_t y_cb, r_cb, q_cb;  // 32-feature blocks of a row in the block layout; 0: row-major
    float inv_so;
    int64_t row0;  // first row of this launch
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
// as rows of any width put them: the hardware takes either as one access
typedef float f32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32_at1 __attribute__((aligned(1)));

template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
// Sum over the wave, in every lane: rotations within 16 lanes, then swaps of
// 16- and 32-lane halves, no LDS.
__device__ __forceinline__ float wave_sum(float v)
{
    v = dpp_add<0x128>(v);  // row_ror:8, 4, 2, 1
    v = dpp_add<0x124>(v);
    v = dpp_add<0x122>(v);
    v = dpp_add<0x121>(v);
    const int b = __float_as_int(v);
    const auto x = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    v = __int_as_float(x[0]) + __int_as_float(x[1]);
    const int c = __float_as_int(v);
    const auto y = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    return __int_as_float(y[0]) + __int_as_float(y[1]);
}

// Sum over the row's W waves. A slot of part is written again only after a
// barrier that follows every read of it.
template <int W>
__device__ __forceinline__ float row_sum(float v, float (*part)[16], int slot, int wave)
{
    v = wave_sum(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) part[slot][wave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += part[slot][i];
    }
    return v;
}

// 4 values of an fp32 row from feature c on (zeros past the row's end). EVEN:
// cols is a multiple of 4.
template <bool EVEN>
__device__ __forceinline__ f32x4 load_f32(const float *row, int32_t c, int32_t cols)
{
    f32x4 v = {0, 0, 0, 0};
    if (EVEN ? c < cols : c + 4 <= cols) {
        v = *reinterpret_cast<const f32x4_at4 *>(row + c);
    } else if (!EVEN) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (c + i < cols) v[i] = row[c + i];
    }
    return v;
}

// 4 codes of row t from feature c on, as the 4 bytes of a word. The block
// layout's rows are whole blocks of 32 features, so a word never leaves them.
template <bool EVEN>
__device__ __forceinline__ uint32_t load_i8(const int8_t *x, int64_t t, int32_t c, int32_t cols, int32_t cb)
{
    if (c >= cols) return 0;
    if (cb) return *reinterpret_cast<const uint32_t *>(x + t16x32_offset(t, c, cb));
    const int8_t *row = x + t * cols;
    if (EVEN || c + 4 <= cols) return *reinterpret_cast<const u32_at1 *>(row + c);
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (c + i < cols) v |= (uint32_t)(uint8_t)row[c + i] << (8 * i);
    return v;
}

__device__ __forceinline__ f32x4 codes_to_f32(uint32_t w, float scale)
{
    return f32x4{(float)(int8_t)w * scale, (float)(int8_t)(w >> 8) * scale, (float)(int8_t)(w >> 16) * scale,
                 (float)(int8_t)(w >> 24) * scale};
}

// A lane's first feature, opaque to the compiler where its pieces are many: it
// would compare every feature with the row's end once and keep the outcomes
// over the whole kernel, more of them than there are registers.
template <int IT>
__device__ __forceinline__ int32_t fresh(int32_t c0)
{
    if constexpr (IT == 16) asm volatile("" : "+v"(c0));
    return c0;
}

template <bool EVEN>
__device__ __forceinline__ void store_f32(float *row, int32_t c, int32_t cols, f32x4 v)
{
    if (EVEN ? c < cols : c + 4 <= cols) {
        store_nt_at4(row + c, __builtin_bit_cast(i32x4, v));
    } else if (!EVEN) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (c + i < cols) row[c + i] = v[i];
    }
}

// Norm of a row in place. Values past the row's end are 0 on entry and unspecified on return.
//
// LayerNorm's deviations are from a mean that carries the roundings of its sum,
// up to a few bits of the row's values. Where the mean is large against the
// spread, that is no longer small (rows of one value, whose deviations are
// nothing else, gave +-1 before gamma where the definition has 0): past a mean of
// 4 deviations, the mean of the deviations is taken off them once more. Ordinary
// rows pay for the question only (summing both at once would cost every row: 2048
// x 768 6.2 us against 5.8, 8192 x 3013 60 against 56).
template <int W, int IT, bool EVEN>
__device__ __forceinline__ void norm_row(f32x4 (&v)[IT], int32_t kind, const float *gamma, const float *beta, float eps,
                                         int32_t c0, int32_t cols, float (*part)[16], int slot, int wave)
{
    constexpr int kStep = 256 * W;
    if (kind == SL_NORM_NONE) return;
    // weights are asked for before the sums, whose latency hides theirs (a lane of 16 pieces has no registers for that)
    constexpr bool kEarly = IT < 16;
    f32x4 g[kEarly ? IT : 1], b[kEarly ? IT : 1];
    const auto weights = [&](int i, int32_t c) {
        g[i] = gamma ? load_f32<EVEN>(gamma, c, cols) : f32x4{1, 1, 1, 1};
        b[i] = beta ? load_f32<EVEN>(beta, c, cols) : f32x4{0, 0, 0, 0};
    };
    if constexpr (kEarly) {
#pragma unroll
        for (int i = 0; i < IT; ++i) weights(i, c0 + i * kStep);
    }
    const float inv_n = 1.0f / (float)cols;
    float mean = 0.0f, s = 0.0f;
    if (kind == SL_NORM_LAYER) {
#pragma unroll
        for (int i = 0; i < IT; ++i) s += (v[i][0] + v[i][1]) + (v[i][2] + v[i][3]);
        mean = row_sum<W>(s, part, slot, wave) * inv_n;
        s = 0.0f;
    }
    const auto centre = [&](float by) {  // takes `by` off and sums the squares
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int32_t c = fresh<IT>(c0) + i * kStep;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[i][j] -= by;
                if (c + (EVEN ? 0 : j) < cols) sq = fmaf(v[i][j], v[i][j], sq);
            }
        }
        return sq;
    };
    float var = row_sum<W>(centre(mean), part, slot + 1, wave) * inv_n + eps;
    if (__any(mean * mean > 16.0f * var)) {  // (the same for every lane of a row)
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int32_t c = fresh<IT>(c0) + i * kStep;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + (EVEN ? 0 : j) < cols) s += v[i][j];
        }
        const float rest = row_sum<W>(s, part, slot + 2, wave) * inv_n;
        var = row_sum<W>(centre(rest), part, slot + 3, wave) * inv_n + eps;
    }
    const float rstd = 1.0f / sqrtf(var);
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        if constexpr (kEarly) {
            v[i] = v[i] * rstd * g[i] + b[i];
        } else {
            const int32_t c = fresh<IT>(c0) + i * kStep;
            v[i] *= rstd;
            if (gamma) v[i] *= load_f32<EVEN>(gamma, c, cols);
            if (beta) v[i] += load_f32<EVEN>(beta, c, cols);
        }
    }
}

// WG = waves of a workgroup: WG / W rows. Rows of three pieces a lane are held to
// 80 registers, six waves a SIMD (82 and five: 8192 x 3013 60 us against 53).
template <int W, int IT, bool EVEN, int WG>
__global__ __launch_bounds__(64 * WG) __attribute__((amdgpu_waves_per_eu(IT == 3 ? 6 : 4)))
void residual_norm_kernel(const NormArgs p)
{
    __shared__ float part[W > 1 ? 8 : 1][16];
    const sl_residual_norm_args &a = p.a;
    constexpr int kStep = 256 * W;
    const int wave = threadIdx.x >> 6;
    const int64_t row = p.row0 + (int64_t)blockIdx.x * (WG / W) + wave / W;
    if (row >= a.rows) return;  // (a whole workgroup where W > 1)
    const int w = wave % W;
    const int32_t cols = a.cols, c0 = (w * 64 + (int)(threadIdx.x & 63)) * 4;
    const bool y8 = a.y_type == SL_ACT_I8, r8 = a.r_type == SL_ACT_I8;
    // the words of a piece as loaded: fp32 values, or codes in the first word
    const auto load = [&](bool codes, const void *x, int32_t c, int32_t cb) {
        if (!codes) return load_f32<EVEN>(reinterpret_cast<const float *>(x) + row * cols, c, cols);
        return f32x4{__uint_as_float(load_i8<EVEN>(reinterpret_cast<const int8_t *>(x), row, c, cols, cb)), 0, 0, 0};
    };
    // and its values: zeros past the row's end, where a word of codes may hold anything
    const auto value = [&](bool codes, f32x4 v, float scale, int32_t c) {
        if (!codes) return v;
        v = codes_to_f32(__float_as_uint(v[0]), scale);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + (EVEN ? 0 : j) >= cols) v[j] = 0.0f;
        return v;
    };
    // (a lane of 16 pieces has no registers for both inputs: it reads r when it needs it. The gate is never read
    // ahead: 49152 x 1024 of channel gates 125 us against 120 for the waves that its registers cost)
    constexpr bool kEarly = IT < 16;
    f32x4 y[IT], x[kEarly ? IT : 1];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int32_t c = fresh<IT>(c0) + i * kStep;
        y[i] = load(y8, a.y, c, p.y_cb);
        if (kEarly && a.r_type != SL_ACT_NONE) x[i] = load(r8, a.r, c, p.r_cb);
    }
#pragma unroll
    for (int i = 0; i < IT; ++i) y[i] = value(y8, y[i], a.y_scale, fresh<IT>(c0) + i * kStep);
    norm_row<W, IT, EVEN>(y, a.post_kind, a.post_gamma, a.post_beta, a.eps, c0, cols, part, 0, w);
    const float gt = a.gate_kind == SL_GATE_TOKEN ? a.gate[row] : 1.0f;
    const float *gr = a.gate_kind == SL_GATE_CHANNEL ? a.gate : a.gate + row * cols;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int32_t c = fresh<IT>(c0) + i * kStep;
        if (a.gate_kind == SL_GATE_TOKEN)
            y[i] *= gt;
        else if (a.gate_kind != SL_GATE_NONE)
            y[i] *= load_f32<EVEN>(gr, c, cols);
        if (a.r_type != SL_ACT_NONE) {
            if constexpr (!kEarly) x[0] = load(r8, a.r, c, p.r_cb);
            y[i] = value(r8, x[kEarly ? i : 0], a.r_scale, c) * a.residual_scale + y[i];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + (EVEN ? 0 : j) >= cols) y[i][j] = 0.0f;
        if (a.h) store_f32<EVEN>(a.h + row * cols, c, cols, y[i]);
    }
    norm_row<W, IT, EVEN>(y, a.norm_kind, a.gamma, a.beta, a.eps, c0, cols, part, 4, w);
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int32_t c = fresh<IT>(c0) + i * kStep;
        if (a.u) store_f32<EVEN>(a.u + row * cols, c, cols, y[i]);
        if (!a.q || c >= cols) continue;
        const uint32_t b = pack_bytes(requant_bits(y[i][0], p.inv_so), requant_bits(y[i][1], p.inv_so),
                                      requant_bits(y[i][2], p.inv_so), requant_bits(y[i][3], p.inv_so));
        if (p.q_cb) {
            *reinterpret_cast<uint32_t *>(a.q + t16x32_offset(row, c, p.q_cb)) = b;
        } else if (EVEN || c + 4 <= cols) {
            *reinterpret_cast<u32_at1 *>(a.q + row * cols + c) = b;
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (c + j < cols) a.q[row * cols + c + j] = (int8_t)(b >> (8 * j));
        }
    }
}

template <int W, int IT, int WG>
sl_status launch_shape(NormArgs p, hipStream_t s)
{
    constexpr int64_t kRows = WG / W, kMostWgs = 0x7fffffff / (64 * WG);  // a launch has less than 2^31 threads
    for (; p.row0 < p.a.rows; p.row0 += kMostWgs * kRows) {
        const dim3 wgs((uint32_t)std::min(kMostWgs, (p.a.rows - p.row0 + kRows - 1) / kRows));
        if (p.a.cols % 4 == 0)
            hipLaunchKernelGGL((residual_norm_kernel<W, IT, true, WG>), wgs, dim3(64 * WG), 0, s, p);
        else
            hipLaunchKernelGGL((residual_norm_kernel<W, IT, false, WG>), wgs, dim3(64 * WG), 0, s, p);
        HIP_TRY(hipGetLastError());
    }
    return SL_OK;
}

}  // namespace

sl_status launch_residual_norm(const sl_residual_norm_args &a, void *stream)
{
    const hipStream_t s = static_cast<hipStream_t>(stream);
    NormArgs p{};
    p.a = a;
    const int32_t cb = (a.cols + 31) / 32;
    const auto tiles = [&](const void *x, int32_t layout) { return x && layout == SL_LAYOUT_T16X32 ? cb : 0; };
    p.y_cb = a.y_type == SL_ACT_I8 ? tiles(a.y, a.y_layout) : 0;
    p.r_cb = a.r_type == SL_ACT_I8 ? tiles(a.r, a.r_layout) : 0;
    p.q_cb = tiles(a.q, a.q_layout);
    p.inv_so = a.q ? 1.0f / a.out_scale : 1.0f;
    if (a.cols <= 256) return launch_shape<1, 1, 4>(p, s);
    if (a.cols <= 512) return launch_shape<1, 2, 4>(p, s);
    // Few rows: a row's chain of loads, sums and stores counts, and four waves shorten it. Up to 2048 rows: 128 x 768 3.2
    // us against 4.0, 1024 x 1024 4.5 against 4.8, 1531 x 1001 with norms on both sides 8.1 against 10.3; 2048 x 768 6.0
    // against 5.8. More: 49152 x 1024 95 against 90, with norms on both sides, int8 y and h kept 146 against 118.
    if (a.rows <= 2048 && a.cols <= 1024) return launch_shape<4, 1, 4>(p, s);
    if (a.cols <= 768) return launch_shape<1, 3, 4>(p, s);
    if (a.cols <= 1024) return launch_shape<1, 4, 4>(p, s);
    if (a.cols <= 2048) return launch_shape<4, 2, 4>(p, s);
    // (8192 x 2894 with four pieces a lane 77 us against 66; 8192 x 4096 on four waves 79 against 77, with norms on both
    // sides and a gate 100 against 90)
    if (a.cols <= 3072) return launch_shape<4, 3, 4>(p, s);
    if (a.cols <= 4096) return launch_shape<8, 2, 8>(p, s);
    if (a.cols <= 16384) return launch_shape<16, 4, 16>(p, s);
    return launch_shape<16, 16, 16>(p, s);
}

}  // namespace sl
