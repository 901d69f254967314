// Rows kept in 8 bits (include/mpcnn.h, mpcnn_packed): blocks of 32 features share a power of two, 2^e, the least for which the block's largest magnitude is
// at most 127 2^e (MPCNN_I8) or 448 2^e (MPCNN_E4M3), and -100 <= e <= 121 or 120 (what is kept reads back finite); a number is kept as x 2^-e, rounded to nearest even (the product is exact).  The scale's
// byte is e + 127; 255 stands for a block with a number that is not finite, and all of it reads as NaN.
//
// A power of two and no finer scale: a number of either kind times its scale has at most 8 significant bits, which is an exact bf16 number (from 2^-109 up, far above
// bf16's smallest), so that matrix products read packed rows without a rounding more.  The price is up to one bit of MPCNN_I8's blocks (their largest number is kept as 64 .. 127).
#pragma once
#include "../../include/mpcnn.h"
#include "any_address.hpp"
#include "lanes.hpp"
#include "ranges.hpp"

namespace mpcnn {

constexpr int kBlock = 32;                 // features of a scale
constexpr int kLeastScale = 127 - 100;     // its byte
constexpr int kMostScaleI = 127 + 121, kMostScaleE = 127 + 120;   // where the kept numbers end at 127 and 240: the next ones read back would be infinite
constexpr unsigned kNaNScale = 255;
typedef unsigned u2 __attribute__((ext_vector_type(2)));

// A packed matrix as kernels see it: [rows][padded] bytes and [rows][padded / 32] scales; padded: features up to whole blocks, zeros behind the last
struct Packed {
    unsigned char *values, *scales;        // null: none
    int kind;                              // mpcnn_packing
};

// The scale's byte of a block whose largest magnitude has the bits `peak` (a NaN's are above infinity's, so it is not passed over)
__device__ __forceinline__ unsigned scale_of(unsigned peak, int kind)
{
    const unsigned field = peak >> 23, mantissa = peak & 0x7fffff;
    if (field == 255) return kNaNScale;
    const int byte = kind == MPCNN_I8 ? (int)field - 6 + (mantissa > 0x7e0000) : (int)field - 8 + (mantissa > 0x600000);   // 127 = 1.984375 2^6, 448 = 1.75 2^8
    const int most = kind == MPCNN_I8 ? kMostScaleI : kMostScaleE;
    return (unsigned)(byte < kLeastScale ? kLeastScale : byte > most ? most : byte);
}
// Eight numbers in 8 bits; nothing of a block that is not finite
__device__ __forceinline__ u2 pack8(v8f v, unsigned scale, int kind)
{
    if (scale == kNaNScale) return u2{0, 0};
    const float up = power_of_two(127 - (int)scale);
    if (scale >= (unsigned)kMostScaleE) {                    // (hardly ever)
        const float end = kind == MPCNN_I8 ? 127.f : 240.f, top = end / up;
#pragma unroll
        for (int z = 0; z < 8; ++z) v[z] = fminf(fmaxf(v[z], -top), top);
    }
    u2 r;
    if (kind == MPCNN_I8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            unsigned w = 0;
#pragma unroll
            for (int z = 3; z >= 0; --z) w = w << 8 | ((unsigned)(int)__builtin_rintf(v[4 * h + z] * up) & 255u);
            r[h] = w;
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * up, v[4 * h + 1] * up, 0, false);
            r[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * up, v[4 * h + 3] * up, w, true);
        }
    }
    return r;
}
__device__ __forceinline__ float scale_value(unsigned scale)      // a byte that no packing leaves is taken as it is
{
    return scale == kNaNScale ? __builtin_nanf("") : scale ? __builtin_bit_cast(float, scale << 23) : 0x1p-127f;
}
__device__ __forceinline__ v8f unpack8(u2 r, unsigned scale, int kind)
{
    const float by = scale_value(scale);
    v8f v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (kind == MPCNN_I8) {
#pragma unroll
            for (int z = 0; z < 4; ++z) v[4 * h + z] = (float)(int)(signed char)(r[h] >> (8 * z) & 255u) * by;
        } else {
            typedef float v2f __attribute__((ext_vector_type(2)));
            const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)r[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)r[h], true);
            v[4 * h] = lo[0] * by; v[4 * h + 1] = lo[1] * by; v[4 * h + 2] = hi[0] * by; v[4 * h + 3] = hi[1] * by;
        }
    }
    return v;
}

// Eight numbers of a row, `at` its first of them, by the 4 lanes side by side that have a block (all of them here, zeros where there is no feature)
__device__ __forceinline__ void pack_store(const Packed& p, long row, int padded, int at, v8f v)
{
    unsigned peak = 0;
#pragma unroll
    for (int z = 0; z < 8; ++z) {
        const unsigned b = bits_of(v[z]) & 0x7fffffffu;
        peak = b > peak ? b : peak;
    }
    const unsigned scale = scale_of(largest4(peak), p.kind);
    *reinterpret_cast<u2*>(p.values + row * padded + at) = pack8(v, scale, p.kind);
    if (at % kBlock == 0) p.scales[row * (padded / kBlock) + at / kBlock] = (unsigned char)scale;
}

}  // namespace mpcnn
