// What attention_run and cache_attention of many queries share on the device: the
// numbers that scores and weights are held as (kernels_attention.hip says why), and
// how operands lie in LDS. Not part of the public ABI.
#pragma once

#include <math.h>

#include <algorithm>

#include "sl_device.h"

namespace sl {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kChunk = SL_KEY_BLOCK;      // keys of a step
constexpr int32_t kMagic = 0x4B400000;    // bits of 1.5 * 2^23
constexpr float kMagicF = 12582912.0f;
// P carries a factor of up to 2^8 (see exponent_of), so that small weights keep more of their bits. A lane's 32
// weights of a chunk then sum to 2^13 at most where m is the maximum; while they sum to less than kMostSum, none is over
// what 16 bits hold.
constexpr float kMostSum = 60000.0f;
// m before the first key: below every score, and close enough that S - m keeps within the offset's 2^22
constexpr int32_t kLowest = -(1 << 21);

// byte offset of feature c of token t
__device__ __forceinline__ int64_t at(int64_t t, int32_t c, int32_t cols, int32_t cb)
{
    return cb ? t16x32_offset(t, c, cb) : t * cols + c;
}

// A lane number that the compiler takes for a new one: addresses made from it
// are not computed before the loop over chunks and kept through it.
__device__ __forceinline__ int here(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}

// 16 bytes a lane to 64 pieces of LDS in order of the lanes, from `to` on; landed once the wave's loads are waited for.
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t x, char *to, uint32_t offset, uint32_t more)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(x, (lds_void *)to, 16, offset, more, 0, 0);
}

// Of the two lanes that hold a query's scores.
__device__ __forceinline__ int pair_max(int v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((int)a[0], (int)a[1]);
}
__device__ __forceinline__ float pair_sum(float v)
{
    const int b = __float_as_int(v);
    const auto a = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return __int_as_float(a[0]) + __int_as_float(a[1]);
}

// Permutations of the 16-byte pieces of a row in LDS. A 16-byte read is served
// 16 lanes at a time, lanes 0-3, 12-15 and 20-27 of each 32 and then the others.
// With a lane a row, these spread each such set of rows over all 64 banks (4.4
// cycles a read, against 8.5 with rows padded by 16 bytes).
template <int N>
__device__ __forceinline__ int kswap(int row)  // key rows of 32 N bytes
{
    return N == 2 ? (row >> 2) & 3 : N == 4 ? (row >> 1) & 7 : (row >> 3) & 1;
}
__device__ __forceinline__ int vswap(int row) { return (row >> 1) & 7; }  // value rows of 128 bytes

// Factor and offset of the exponential's argument for scores that `scale` multiplies.
struct Exponent {
    float c2, k2;
};
inline Exponent exponent_of(double scale)
{
    Exponent x;
    // log2 units a whole number of S is worth, rounded to 22 bits: times 1.5 * 2^23 it is then a float itself,
    // and the exponent of P loses nothing to that offset
    // (not 0: minus infinity times it has to stay what it is)
    const double c2 = std::max(scale * 1.4426950408889634, 1e-30);
    int e = 0;
    const double frac = frexp(c2, &e);
    x.c2 = (float)ldexp(nearbyint(ldexp(frac, 22)), e - 22);
    // P's factor is 2^7, and past 2^24 what the offset can take without losing a bit: multiples of 2, 4 and 8 up to 2^27,
    // then nothing (weights of neighbouring scores differ by 10 octaves and more there, at 2^24 by 1.3)
    const float offset = kMagicF * x.c2;
    const float factor = offset < 0x1p24f   ? 7.0f
                         : offset < 0x1p25f ? 6.0f
                         : offset < 0x1p26f ? 4.0f
                         : offset < 0x1p27f ? 8.0f
                                            : 0.0f;
    x.k2 = factor - offset;
    return x;
}

}  // namespace sl
