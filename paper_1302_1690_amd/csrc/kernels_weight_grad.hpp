// The gradient of a linear layer's weights from rows kept in 8 bits (weight_grad.hip): dw[o][f] = sum over the rows n of dy[n][o] x[n][f].
//
// Products on v_mfma_f32_32x32x16_bf16, sums in fp32.  x in 8 bits times its block's power of two is an exact bf16 number (packed.hpp); bf16 dy is taken as it
// is, fp32 dy as three bf16 parts (24 bits, its exponents as they are), whose products are added up, the smallest first: nothing is rounded but the sums and the result.
//
// A workgroup computes a tile of 32 WM MT x 32 WN NT results, each wave MT x NT of the instruction's.  Both operands have the summed index as the rows of memory;
// blocks of KB rows are fetched into registers while the block before is multiplied, and lie in LDS as they do in memory, as bf16: x is widened on its way
// there, once per workgroup.  The instruction wants 8 rows of one column per lane: ds_read_b64_tr_b16 turns 4 rows x 16 columns around within 16 lanes (lane r
// names 4 columns, r % 4, of row r / 4 and receives column r of all 4).  The 64-byte groups of a row lie permuted by the row's number, on different banks.
#pragma once
#include "packed.hpp"

namespace mpcnn {

struct WeightGradArgs {
    const void* dy;
    long dy_pitch;
    Packed x;
    int N, M, D, padded;                   // rows, outputs, features
    int blocks, per_split, splits;         // along the rows: in all, of a workgroup
    int tiles_m, tiles_n;
    void* dw;                              // [M][D]
    int dw_bf16;
    float* part;                           // [splits][M][D]: partial sums instead
};

typedef __bf16 g_bf16x8 __attribute__((ext_vector_type(8)));
typedef short g_s4 __attribute__((ext_vector_type(4)));
typedef unsigned g_u4 __attribute__((ext_vector_type(4)));

// 8 numbers of packed rows as bf16 (exact)
__device__ __forceinline__ g_bf16x8 widen8(u2 r, unsigned scale, int kind) { return __builtin_convertvector(unpack8(r, scale, kind), g_bf16x8); }

template <typename T, int WM, int WN, int MT, int NT, int KB>
__global__ __launch_bounds__(64 * WM * WN) void weight_grad_kernel(WeightGradArgs a)
{
    constexpr int BM = 32 * WM * MT, BN = 32 * WN * NT, kThreads = 64 * WM * WN;
    constexpr int P = sizeof(T) == 4 ? 3 : 1;            // parts of dy
    constexpr int kARow = 2 * BM, kBRow = 2 * BN;        // bytes
    constexpr int kPart = KB * kARow, kStage = P * kPart + KB * kBRow;
    constexpr int AI = KB * BM / 8 / kThreads, BI = KB * BN / 16 / kThreads;
    static_assert(AI * 8 * kThreads == KB * BM && BI * 16 * kThreads == KB * BN, "the threads share a block evenly");
    extern __shared__ __attribute__((aligned(256))) char lds_raw[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;

    // ---- the workgroup's tile: the XCDs (workgroups go to them in turn) take stretches of the tiles, in groups of 8 tiles along m
    const int tiles = a.tiles_m * a.tiles_n, all = tiles * a.splits, each = (all + 7) / 8;
    const int t = ((int)blockIdx.x % 8) * each + (int)blockIdx.x / 8;
    if ((int)blockIdx.x / 8 >= each || t >= all) return;
    const int split = t / tiles, tt = t - split * tiles;
    const int group = tt / (8 * a.tiles_n), in = tt - group * 8 * a.tiles_n;
    const int deep = a.tiles_m - 8 * group < 8 ? a.tiles_m - 8 * group : 8;
    const int tn = in / deep, tm = 8 * group + in - tn * deep;
    const int m0 = tm * BM, n0 = tn * BN;
    const int first = split * a.per_split, count = a.blocks - first < a.per_split ? a.blocks - first : a.per_split;

    Raw8<T> ra[AI];
    g_u4 rb[BI];
    unsigned rs[BI];
    auto fetch = [&](int block) {
        const long k0 = (long)(first + block) * KB;
#pragma unroll
        for (int i = 0; i < AI; ++i) {
            const int q = tid + kThreads * i, k = q / (BM / 8), at = m0 + 8 * (q % (BM / 8));
            if (k0 + k < a.N && at < a.M) ra[i] = raw8_of((const T*)a.dy + (k0 + k) * a.dy_pitch, at, a.M);
            else ra[i] = Raw8<T>{};
        }
#pragma unroll
        for (int i = 0; i < BI; ++i) {
            const int q = tid + kThreads * i, k = q / (BN / 16), at = n0 + 16 * (q % (BN / 16));
            rb[i] = g_u4{0, 0, 0, 0};
            rs[i] = 127;
            if (k0 + k < a.N && at < a.padded) {
                rb[i] = *reinterpret_cast<const g_u4*>(a.x.values + (k0 + k) * a.padded + at);
                rs[i] = a.x.scales[(k0 + k) * (a.padded / kBlock) + at / kBlock];
            }
        }
    };
    auto stage = [&](char* to) {
#pragma unroll
        for (int i = 0; i < AI; ++i) {
            const int q = tid + kThreads * i, k = q / (BM / 8), p = q % (BM / 8);
            char* const at = to + k * kARow + 16 * (p ^ 4 * (k & 3));
            if constexpr (P == 1) {
                *reinterpret_cast<decltype(ra[i].a)*>(at) = ra[i].a;
            } else {
                v8f v = widen(ra[i]);
#pragma unroll
                for (int z = 0; z < P; ++z) {
                    const g_bf16x8 h = __builtin_convertvector(v, g_bf16x8);
                    *reinterpret_cast<g_bf16x8*>(at + z * kPart) = h;
                    v -= __builtin_convertvector(h, v8f);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BI; ++i) {
            const int q = tid + kThreads * i, k = q / (BN / 16), p = 2 * (q % (BN / 16));
            char* const row = to + P * kPart + k * kBRow;
            *reinterpret_cast<g_bf16x8*>(row + 16 * (p ^ 4 * (k & 3))) = widen8(u2{rb[i][0], rb[i][1]}, rs[i], a.x.kind);
            *reinterpret_cast<g_bf16x8*>(row + 16 * ((p + 1) ^ 4 * (k & 3))) = widen8(u2{rb[i][2], rb[i][3]}, rs[i], a.x.kind);
        }
    };

    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // lane l names 4 columns of row 8 (l / 32) + (l % 16) / 4 of the step's 16, and of the row 4 on
    const int row = lane & 31, half = lane >> 5, turn = (lane & 15) >> 2, of_row = 8 * half + turn, of_col = 32 * (lane >> 4 & 1) + 8 * (lane & 3);
    int at_a[MT], at_b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) at_a[i] = of_row * kARow + of_col + 64 * ((MT * wm + i) ^ turn);
#pragma unroll
    for (int j = 0; j < NT; ++j) at_b[j] = P * kPart + of_row * kBRow + of_col + 64 * ((NT * wn + j) ^ turn);
    auto read = [&](const char* at, int on) {            // 8 rows, the second 4 of them `on` bytes behind
        using Lds = __attribute__((address_space(3))) g_s4*;
        const g_s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + on));
        return __builtin_bit_cast(g_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto multiply = [&](const char* from) {
#pragma unroll
        for (int s = 0; s < KB / 16; ++s) {
            g_bf16x8 x[P][MT], y[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) y[j] = read(from + at_b[j] + 16 * s * kBRow, 4 * kBRow);
#pragma unroll
            for (int z = P - 1; z >= 0; --z) {
#pragma unroll
                for (int i = 0; i < MT; ++i) x[z][i] = read(from + z * kPart + at_a[i] + 16 * s * kARow, 4 * kARow);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[z][i], y[j], acc[i][j], 0, 0, 0);
            }
        }
    };

    if (count > 0) fetch(0);
    for (int b = 0; b < count; ++b) {
        char* const now = lds_raw + (b & 1) * kStage;
        stage(now);
        __syncthreads();
        if (b + 1 < count) fetch(b + 1);
        multiply(now);
    }

#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = n0 + 32 * (NT * wn + j) + row;
            if (n >= a.D) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = m0 + 32 * (MT * wm + i) + 8 * (r >> 2) + 4 * half + (r & 3);
                if (m >= a.M) continue;
                const long at = (long)m * a.D + n;
                if (a.part) a.part[(long)split * a.M * a.D + at] = acc[i][j][r];
                else if (a.dw_bf16) ((bf16*)a.dw)[at] = (bf16)acc[i][j][r];
                else ((float*)a.dw)[at] = acc[i][j][r];
            }
        }
}

// The splits' sums, in their order; without splits, zeros
__global__ __launch_bounds__(256) void weight_grad_sum_kernel(const float* part, int splits, long n, void* out, int out_bf16)
{
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) {
        float s = 0.f;
        for (int z = 0; z < splits; ++z) s += part[z * n + i];
        if (out_bf16) ((bf16*)out)[i] = (bf16)s;
        else ((float*)out)[i] = s;
    }
}

}  // namespace mpcnn
