// Root-mean-square norm of rows of features, its gradients, and rows in 8 bits (rows_norm.hip).
//
//   h = x + residual,  rstd = 1 / sqrt(mean over the features of h^2 + eps),  y = h rstd gain
//   u = dy gain, c = mean of u h rstd:  dx = dh + rstd (u - h rstd c),  dgain = sum over the rows of dy h rstd
//
// Bound by memory: every matrix goes by once.  A row lies in the registers of the lanes that share it (8 features a lane and piece): 16 lanes up to 256
// features, a wave up to 1024, a workgroup of 256 or 1024 beyond, so the second use of its numbers is not read again.  A workgroup goes through rows
// and keeps the gain in registers (with bf16 rows it has twice their bytes).  The next row's numbers are fetched before this one's sum is known.
// The gain's gradient: every lane adds up its features' share over its rows, workgroups leave one share each, which a launch of its own adds in order.
// 16384 x 4096 bf16: the norm with the residual, both sums and two 8-bit outputs, 542 MB, 113 us (4.8 TB/s, a large copy's rate); gradients from 8 bits with dh, 472 MB, 91 us and 6 for the
// gain's shares; into 8 bits 40 us, back 32.  Workgroups of a backward call: two, three, four, six a compute unit 97, 98, 110, 105 us, with 688 features 32, 30, 33, 32.
#pragma once
#include <type_traits>

#include "packed.hpp"

namespace mpcnn {

struct NormArgs {
    const void *x, *residual;
    long x_pitch, residual_pitch;
    const float* gain;
    long rows;
    int D, padded;
    float eps;
    void *y, *h;
    long y_pitch, h_pitch;
    Packed y_packed, h_packed;
    float* rstd;
};

struct NormBackArgs {
    const void *dy, *h, *dh;
    long dy_pitch, h_pitch, dh_pitch;
    Packed h_packed;
    const float *gain, *rstd;
    long rows;
    int D, padded;
    void* dx;
    long dx_pitch;
    float* part;                           // [workgroups][D]: shares of dgain (one workgroup: dgain itself), or null
};

constexpr int threads_of(int lanes) { return lanes > 256 ? lanes : 256; }

// The sum over the lanes that share a row, in all of them; `flip` is another buffer from one call to the next, so that one barrier is enough
template <int LANES, int N>
__device__ __forceinline__ void sum_row(float (&v)[N], float (*red)[N][16], int flip)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = LANES == 16 ? sum16(v[i]) : sum64(v[i]);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[flip][i][wave] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = red[flip][i][0];
#pragma unroll
            for (int w = 1; w < W; ++w) s += red[flip][i][w];
            v[i] = s;
        }
    }
}

// 1 / sqrt(mean + eps) of a row's squares (`mean` with eps, in all lanes that share the row).  Where fp32 does not hold their sum, or too few of their bits, again(by) is the sum of the squares of
// the row's numbers times a power of two, which changes no bits: numbers up to 2^128 times 2^-80 (sum at most 2^96 2^20), or, where the mean is below 2^-100, times 2^100 (2^120; the least number, 2^-149,
// leaves 2^-98).
constexpr float kLeastMean = 0x1p-100f, kMostMean = 3.4028234663852886e38f;
template <typename F>
__device__ __forceinline__ float norm_rstd(float mean, int features, float eps, F again)
{
    if (mean >= kLeastMean && mean <= kMostMean) return 1.f / sqrtf(mean);
    const float by = mean > 1.f ? 0x1p-80f : 0x1p100f;   // (hardly ever)
    return by / sqrtf(again(by) / (float)features + eps * by * by);
}

template <typename T>
__device__ __forceinline__ void norm_store(const NormArgs& a, long n, int at, v8f h, v8f gain, float rstd)
{
    if (a.h) store8_of((T*)a.h + n * a.h_pitch, at, a.D, h);
    if (a.h_packed.values) pack_store(a.h_packed, n, a.padded, at, h);
    if (!a.y && !a.y_packed.values) return;
    v8f y;
#pragma unroll
    for (int z = 0; z < 8; ++z) y[z] = h[z] * rstd * gain[z];
    if (a.y) store8_of((T*)a.y + n * a.y_pitch, at, a.D, y);
    if (a.y_packed.values) pack_store(a.y_packed, n, a.padded, at, y);
}

// LANES share a row of at most 8 LANES E features
template <typename T, int LANES, int E>
__global__ __launch_bounds__(threads_of(LANES)) void rows_norm_kernel(NormArgs a)
{
    constexpr int kSlots = threads_of(LANES) / LANES;
    __shared__ float red[2][1][16];
    const int t = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    int at[E];
    v8f gain[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        at[e] = 8 * (t + LANES * e);
        gain[e] = at[e] < a.D ? load8_of(a.gain, at[e], a.D) : v8f{};
    }
    Raw8<T> x[E], r[E];
    auto fetch = [&](long n) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (at[e] >= a.D) continue;
            x[e] = raw8_of((const T*)a.x + n * a.x_pitch, at[e], a.D);
            if (a.residual) r[e] = raw8_of((const T*)a.residual + n * a.residual_pitch, at[e], a.D);
        }
    };
    long n = (long)blockIdx.x * kSlots + slot;
    const long step = (long)gridDim.x * kSlots;
    if (n < a.rows) fetch(n);
    for (int flip = 0; n < a.rows; n += step, flip ^= 1) {
        v8f h[E];
        float sum[1] = {0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
            h[e] = at[e] < a.D ? widen(x[e]) : v8f{};
            if (a.residual && at[e] < a.D) h[e] += widen(r[e]);
#pragma unroll
            for (int z = 0; z < 8; ++z) sum[0] = fmaf(h[e][z], h[e][z], sum[0]);
        }
        if (n + step < a.rows) fetch(n + step);
        sum_row<LANES>(sum, red, flip);
        const float rstd = norm_rstd(sum[0] / (float)a.D + a.eps, a.D, a.eps, [&](float by) {
            float far[1] = {0.f};
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int z = 0; z < 8; ++z) far[0] = fmaf(h[e][z] * by, h[e][z] * by, far[0]);
            sum_row<LANES>(far, red, flip ^= 1);
            return far[0];
        });
        if (a.rstd && t == 0) a.rstd[n] = rstd;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at[e] < a.padded) norm_store<T>(a, n, at[e], h[e], gain[e], rstd);
    }
}

// Rows that no workgroup's registers hold: read twice
template <typename T>
__global__ __launch_bounds__(1024) void rows_norm_long_kernel(NormArgs a)
{
    __shared__ float red[2][1][16];
    int flip = 0;
    for (long n = blockIdx.x; n < a.rows; n += gridDim.x, flip ^= 1) {
        const T* const x = (const T*)a.x + n * a.x_pitch;
        const T* const r = a.residual ? (const T*)a.residual + n * a.residual_pitch : nullptr;
        auto row = [&](int at) {
            v8f h = at < a.D ? load8_of(x, at, a.D) : v8f{};
            if (r && at < a.D) h += load8_of(r, at, a.D);
            return h;
        };
        float sum[1] = {0.f};
        for (int at = 8 * threadIdx.x; at < a.D; at += 8 * 1024) {
            const v8f h = row(at);
#pragma unroll
            for (int z = 0; z < 8; ++z) sum[0] = fmaf(h[z], h[z], sum[0]);
        }
        sum_row<1024>(sum, red, flip);
        const float rstd = norm_rstd(sum[0] / (float)a.D + a.eps, a.D, a.eps, [&](float by) {
            float far[1] = {0.f};
            for (int at = 8 * threadIdx.x; at < a.D; at += 8 * 1024) {
                const v8f h = row(at);
#pragma unroll
                for (int z = 0; z < 8; ++z) far[0] = fmaf(h[z] * by, h[z] * by, far[0]);
            }
            sum_row<1024>(far, red, flip ^= 1);
            return far[0];
        });
        if (a.rstd && threadIdx.x == 0) a.rstd[n] = rstd;
        for (int at = 8 * threadIdx.x; at < a.padded; at += 8 * 1024)
            norm_store<T>(a, n, at, row(at), at < a.D ? load8_of(a.gain, at, a.D) : v8f{}, rstd);
    }
}

// What a row's gradient needs of 8 features; a row whose dy is zero throughout adds nothing, whatever h holds
struct NormPiece { v8f dy, unit; };
__device__ __forceinline__ NormPiece norm_piece(v8f dy, v8f h, v8f gain, float rstd, float (&sum)[2])
{
    NormPiece p{dy, h * rstd};
    unsigned some = 0;
#pragma unroll
    for (int z = 0; z < 8; ++z) {
        sum[0] = fmaf(dy[z] * gain[z], p.unit[z], sum[0]);
        some |= bits_of(dy[z]) & 0x7fffffffu;
    }
    if (some) sum[1] = 1.f;
    return p;
}

template <typename T, int LANES, int E, bool PACKED>
__global__ __launch_bounds__(threads_of(LANES)) void rows_norm_back_kernel(NormBackArgs a)
{
    constexpr int kThreads = threads_of(LANES), kSlots = kThreads / LANES;
    __shared__ float red[2][2][16];
    __shared__ __attribute__((aligned(32))) float shares[kSlots > 1 ? kSlots * LANES * 8 * E : 1];
    const int t = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    int at[E];
    v8f gain[E], dgain[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        at[e] = 8 * (t + LANES * e);
        gain[e] = at[e] < a.D ? load8_of(a.gain, at[e], a.D) : v8f{};
        dgain[e] = v8f{};
    }
    Raw8<T> dy[E], more[E];
    std::conditional_t<PACKED, u2, Raw8<T>> h[E];
    unsigned char scale[E];
    float rstd = 0.f;
    auto fetch = [&](long n) {
        rstd = a.rstd[n];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (at[e] >= a.D) continue;
            dy[e] = raw8_of((const T*)a.dy + n * a.dy_pitch, at[e], a.D);
            if constexpr (PACKED) {
                h[e] = *reinterpret_cast<const u2*>(a.h_packed.values + n * a.padded + at[e]);
                scale[e] = a.h_packed.scales[n * (a.padded / kBlock) + at[e] / kBlock];
            } else {
                h[e] = raw8_of((const T*)a.h + n * a.h_pitch, at[e], a.D);
            }
            if (a.dh) more[e] = raw8_of((const T*)a.dh + n * a.dh_pitch, at[e], a.D);
        }
    };
    long n = (long)blockIdx.x * kSlots + slot;
    const long step = (long)gridDim.x * kSlots;
    if (n < a.rows) fetch(n);
    for (int flip = 0; n < a.rows; n += step, flip ^= 1) {
        // Registers for a row's pieces, and for the next row's numbers beside them; else the pieces are made again (more waves instead: 8000 x 4000 fp32 110 us, 113 kept; bf16 16384 x 4096 103, 98 kept)
        constexpr bool kKeep = E < 2 || (E < 4 && sizeof(T) == 2);
        float sum[2] = {0.f, 0.f};
        const float by = rstd;
        auto piece = [&](int e, float (&to)[2]) {
            v8f of;
            if constexpr (PACKED) of = unpack8(h[e], scale[e], a.h_packed.kind);
            else of = widen(h[e]);
            return norm_piece(widen(dy[e]), of, gain[e], by, to);
        };
        NormPiece p[kKeep ? E : 1];
        v8f add[kKeep ? E : 1];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (kKeep) { p[e] = NormPiece{}; add[e] = v8f{}; }
            if (at[e] >= a.D) continue;
            const NormPiece q = piece(e, sum);
            if constexpr (kKeep) {
                p[e] = q;
                if (a.dh) add[e] = widen(more[e]);
            }
        }
        if (kKeep && n + step < a.rows) fetch(n + step);
        sum_row<LANES>(sum, red, flip);
        const bool some = sum[1] != 0.f;
        const float c = some ? sum[0] / (float)a.D : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            NormPiece q{};
            v8f dx{};
            if constexpr (kKeep) {
                q = p[e];
                dx = add[e];
            } else if (at[e] < a.D) {
                float unused[2] = {0.f, 0.f};
                q = piece(e, unused);
                if (a.dh) dx = widen(more[e]);
            }
            if (some) {
#pragma unroll
                for (int z = 0; z < 8; ++z) {
                    dx[z] = fmaf(by, fmaf(-q.unit[z], c, q.dy[z] * gain[e][z]), dx[z]);
                    dgain[e][z] = fmaf(q.dy[z], q.unit[z], dgain[e][z]);
                }
            }
            if (a.dx && at[e] < a.D) store8_of((T*)a.dx + n * a.dx_pitch, at[e], a.D, dx);
        }
        if (!kKeep && n + step < a.rows) fetch(n + step);
    }
    if (!a.part) return;
    float* const part = a.part + (long)blockIdx.x * a.D;
    if constexpr (kSlots > 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) *reinterpret_cast<v8f*>(shares + slot * (LANES * 8 * E) + at[e]) = dgain[e];
        __syncthreads();
        for (int i = threadIdx.x; i < a.D; i += kThreads) {
            float s = shares[i];
#pragma unroll
            for (int k = 1; k < kSlots; ++k) s += shares[k * (LANES * 8 * E) + i];
            part[i] = s;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at[e] < a.D) store8_of(part, at[e], a.D, dgain[e]);
    }
}

// Rows that no workgroup's registers hold: read twice, the shares of dgain kept in memory
template <typename T, bool PACKED>
__global__ __launch_bounds__(1024) void rows_norm_back_long_kernel(NormBackArgs a)
{
    __shared__ float red[2][2][16];
    float* const part = a.part ? a.part + (long)blockIdx.x * a.D : nullptr;
    int flip = 0;
    bool first = true;
    for (long n = blockIdx.x; n < a.rows; n += gridDim.x, flip ^= 1) {
        const float rstd = a.rstd[n];
        auto piece = [&](int at, float (&sum)[2]) {
            const v8f dy = load8_of((const T*)a.dy + n * a.dy_pitch, at, a.D);
            v8f h;
            if constexpr (PACKED)
                h = unpack8(*reinterpret_cast<const u2*>(a.h_packed.values + n * a.padded + at), a.h_packed.scales[n * (a.padded / kBlock) + at / kBlock],
                            a.h_packed.kind);
            else h = load8_of((const T*)a.h + n * a.h_pitch, at, a.D);
            return norm_piece(dy, h, load8_of(a.gain, at, a.D), rstd, sum);
        };
        float sum[2] = {0.f, 0.f};
        for (int at = 8 * threadIdx.x; at < a.D; at += 8 * 1024) piece(at, sum);
        sum_row<1024>(sum, red, flip);
        const bool some = sum[1] != 0.f;
        const float c = some ? sum[0] / (float)a.D : 0.f;
        for (int at = 8 * threadIdx.x; at < a.D; at += 8 * 1024) {
            float unused[2] = {0.f, 0.f};
            const NormPiece p = piece(at, unused);
            const v8f gain = load8_of(a.gain, at, a.D);
            v8f dx = a.dh ? load8_of((const T*)a.dh + n * a.dh_pitch, at, a.D) : v8f{};
            v8f dgain = part && !first ? load8_of(part, at, a.D) : v8f{};
            if (some) {
#pragma unroll
                for (int z = 0; z < 8; ++z) {
                    dx[z] = fmaf(rstd, fmaf(-p.unit[z], c, p.dy[z] * gain[z]), dx[z]);
                    dgain[z] = fmaf(p.dy[z], p.unit[z], dgain[z]);
                }
            }
            if (a.dx) store8_of((T*)a.dx + n * a.dx_pitch, at, a.D, dx);
            if (part) store8_of(part, at, a.D, dgain);
        }
        first = false;
    }
}

// dgain: the workgroups' shares added up, 16 features a workgroup, each by 64 threads over a stretch of the shares
constexpr int kGainColumns = 16, kGainStretches = 64;
__global__ __launch_bounds__(kGainColumns * kGainStretches) void norm_gain_kernel(const float* part, int parts, int D, float* dgain)
{
    __shared__ float red[kGainStretches][kGainColumns + 1];
    const int c = threadIdx.x % kGainColumns, q = threadIdx.x / kGainColumns, at = blockIdx.x * kGainColumns + c;
    float s = 0.f;
    if (at < D) {
#pragma unroll 8
        for (int g = q; g < parts; g += kGainStretches) s += part[(long)g * D + at];
    }
    red[q][c] = s;
    __syncthreads();
    if (q == 0 && at < D) {
#pragma unroll
        for (int k = 1; k < kGainStretches; ++k) s += red[k][c];
        dgain[at] = s;
    }
}

// Rows into 8 bits and back.  A workgroup has some rows' pieces of 8 features, a thread kPieces of them at a time (all fetched before the first is packed): 4 lanes side by
// side have a block (a row is whole blocks, and the loop's step whole waves).
struct PackArgs {
    const void* x;
    long x_pitch;
    void* out;                             // unpacking
    long out_pitch;
    Packed packed;
    long rows;
    int D, padded, each;                   // each: rows of a workgroup
};
constexpr int kPieces = 4;
// fetch(k, row, at) for each of the thread's next pieces, and then use(k, row, at)
template <typename F, typename G>
__device__ __forceinline__ void each_piece(const PackArgs& a, F fetch, G use)
{
    const int pieces = a.padded / 8;
    const long first = (long)blockIdx.x * a.each;
    const int rows = (int)(a.rows - first < a.each ? a.rows - first : a.each), all = rows * pieces;
    const float by = 1.f / (float)pieces;
    for (int i = threadIdx.x; i < all; i += 256 * kPieces) {
        int r[kPieces], at[kPieces];
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            r[k] = (int)(((float)(i + 256 * k) + 0.5f) * by);          // (all < 2^18: exact)
            at[k] = 8 * (i + 256 * k - r[k] * pieces);
            if (i + 256 * k < all) fetch(k, first + r[k], at[k]);
        }
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (i + 256 * k < all) use(k, first + r[k], at[k]);
    }
}
template <typename T>
__global__ __launch_bounds__(256) void rows_pack8_kernel(PackArgs a)
{
    Raw8<T> x[kPieces];
    each_piece(a, [&](int k, long n, int at) { if (at < a.D) x[k] = raw8_of((const T*)a.x + n * a.x_pitch, at, a.D); },
               [&](int k, long n, int at) { pack_store(a.packed, n, a.padded, at, at < a.D ? widen(x[k]) : v8f{}); });
}
template <typename T>
__global__ __launch_bounds__(256) void rows_unpack8_kernel(PackArgs a)
{
    u2 x[kPieces];
    unsigned char scale[kPieces];
    each_piece(a,
               [&](int k, long n, int at) {
                   x[k] = *reinterpret_cast<const u2*>(a.packed.values + n * a.padded + at);
                   scale[k] = a.packed.scales[n * (a.padded / kBlock) + at / kBlock];
               },
               [&](int k, long n, int at) {
                   if (at < a.D) store8_of((T*)a.out + n * a.out_pitch, at, a.D, unpack8(x[k], scale[k], a.packed.kind));
               });
}

}  // namespace mpcnn
