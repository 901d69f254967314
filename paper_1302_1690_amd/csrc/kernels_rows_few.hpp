// The class layer's gradients on at most sixteen rows of features, and scores on at most twelve (class_rows.hip): bound by the passes over the
// class weights (read for the scores, read for the rows' gradient, their own gradient written), so everything is done on the vector
// ALU in fp32, with 128-bit fetches and stores at whatever address the numbers have, and nothing is fetched for rows that do not exist.
// A kernel instance per number of rows.
//
//   rows_few_scores   16 lanes share a class, 8 features a lane and step; a group has 4 classes at once, so that a row's features, which
//                     every group reads from LDS, are used 4 times.  64 classes per round of a workgroup; scores stored [class][row];
//                     per workgroup and row the largest and the sum of exponentials of all its classes.  (The matrix instruction's
//                     scores, kernels_rows_direct.hpp, fetch 16 bytes of each of 32 classes at once and reach 2.1-2.9 TB/s on large weights, this
//                     kernel up to 5; it has less to do at once with few classes, and more arithmetic per row.  us, here / there: 1 x
//                     4096 x 128000 fp32 404 / 729, bf16 213 / 360; 1 x 1000 x 16000 fp32 20 / 24, bf16 15 / 14; 8 x 1024 x 32000 fp32 33 / 39.  Whole calls of the loss:
//                     fp32 12 x 2912 x 73000 270 / 460, 3 x 2912 x 10000 40 / 58, 8 x 1000 x 10000 34 / 31; bf16 3 x 2912 x 73000 119 / 220, 3 x 2912 x 25000
//                     45 / 49, 12 x 2912 x 73000 217 / 242, 8 x 2912 x 25000 59 / 49, 12 x 2913 x 73000 220 / 353.)
//   rows_few_grads    a thread keeps 8 features (4 with more than eight rows) of every row and their gradients over a stretch of the classes:
//                     one fetch of the class's weights, as many multiplications per row for dx and for dw, one store.  5 x 1000 x 30011 bf16
//                     30 us, 4.0 TB/s of weights read and gradients written.
//   rows_few_sum      adds the workgroups' shares of dx, in a fixed order.
#pragma once
#include "any_address.hpp"
#include "rows_few.hpp"

namespace mpcnn {

// The sum over 16 lanes side by side, in all of them
template <int CTRL>
__device__ __forceinline__ float add_moved(float s)
{
    return s + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, s), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float s)
{
    s = add_moved<0x128>(s);   // row_ror:8, 4, 2, 1
    s = add_moved<0x124>(s);
    s = add_moved<0x122>(s);
    return add_moved<0x121>(s);
}

template <typename T, int NR>
__global__ __launch_bounds__(kFewThreads) void rows_few_scores_kernel(FewArgs a)
{
    constexpr int C = 4;                         // classes of a group of 16 lanes
    constexpr int kFewSteps = NR <= 8 ? 8 : 4;   // of 128 features, whose rows LDS holds at once
    constexpr float kNone = -__builtin_inff();
    __shared__ float sc[NR][kFewRound];
    __shared__ __attribute__((aligned(32))) float xl[NR][128 * kFewSteps];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = tid & 15, group = tid >> 4;
    const T* const x = (const T*)a.x;
    constexpr int NW = (NR + 3) / 4;             // rows whose statistics a wave keeps
    float top[NW], sum[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) { top[i] = kNone; sum[i] = 0.f; }
    const long begin = (long)blockIdx.x * a.each, end = begin + a.each < a.V ? begin + a.each : a.V;
    const int steps = (a.D + 127) / 128, whole = a.D / 128;
    for (long v0 = begin; v0 < end; v0 += kFewRound) {
        float acc[C][NR];
        const T* w[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const long v = v0 + group * C + c;
            w[c] = (const T*)a.w + (v < end ? v : end - 1) * a.w_pitch;
#pragma unroll
            for (int n = 0; n < NR; ++n) acc[c][n] = 0.f;
        }
        // steps of 128 features, the weights of the next two fetched before a step's products
        Raw8<T> u[2][C];
        auto fetch = [&](int s, Raw8<T> (&u)[C]) {
            if (s < whole) {
#pragma unroll
                for (int c = 0; c < C; ++c) u[c] = raw8(w[c] + 128 * s + 8 * l16);
            } else if (s < steps) {
#pragma unroll
                for (int c = 0; c < C; ++c) u[c] = raw8_of(w[c], 128 * s + 8 * l16, a.D);
            }
        };
        fetch(0, u[0]);
        fetch(1, u[1]);
        auto step = [&](int s, Raw8<T> (&u)[C]) {
            if (s % kFewSteps == 0 && (steps > kFewSteps || v0 == begin)) {   // the rows' next features into LDS
                __syncthreads();
#pragma unroll
                for (int n = 0; n < NR; ++n)
                    for (int i = 8 * tid; i < 128 * kFewSteps; i += 8 * kFewThreads)
                        if (128 * s + i < a.D) *reinterpret_cast<v8f*>(xl[n] + i) = load8_of(x + n * a.x_pitch, 128 * s + i, a.D);
                        else *reinterpret_cast<v8f*>(xl[n] + i) = v8f{};
                __syncthreads();
            }
            v8f v[C];
#pragma unroll
            for (int c = 0; c < C; ++c) v[c] = widen(u[c]);
            fetch(s + 2, u);
            const int at = 128 * (s % kFewSteps) + 8 * l16;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const v8f y = *reinterpret_cast<const v8f*>(xl[n] + at);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int z = 0; z < 8; ++z) acc[c][n] = fmaf(v[c][z], y[z], acc[c][n]);
            }
        };
        for (int s = 0; s < steps; s += 2) {
            step(s, u[0]);
            if (s + 1 < steps) step(s + 1, u[1]);
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                float s = acc[c][n];
                s = sum16(s);
                if (l16 == (c * NR + n) % 16) sc[n][group * C + c] = s;
            }
        __syncthreads();
        const long v = v0 + lane;
        const float b = v < end && a.bias ? a.bias[v] : 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int n = wave + 4 * i;
            if (n >= NR) continue;               // (uniform)
            const float s = v < end ? sc[n][lane] + b : kNone;
            if (v < end) {
                if (a.scores) a.scores[v * a.score_row + n] = s;
                if (v == a.mask.labels[n]) a.label_score[n] = s;
            }
            // every lane keeps its own classes' statistics until the end
            const float t = fmaxf(top[i], s), base = t == kNone ? 0.f : t;
            sum[i] = sum[i] * __expf(top[i] - base) + __expf(s - base);
            top[i] = t;
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        const int n = wave + 4 * i;
        if (n >= NR) continue;
        float t = top[i], s = sum[i];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const float ot = __shfl_xor(t, o, 64), os = __shfl_xor(s, o, 64);
            const float m = fmaxf(t, ot), base = m == kNone ? 0.f : m;
            s = s * __expf(t - base) + os * __expf(ot - base);
            t = m;
        }
        if (lane == 0) a.stats[(long)blockIdx.x * a.N + n] = float2{t, s};
    }
}

template <typename T, int NR>
__global__ __launch_bounds__(kFewThreads) void rows_few_grads_kernel(FewArgs a)
{
    constexpr int E = few_columns(NR);
    typedef float vef __attribute__((ext_vector_type(E)));
    __shared__ float delta[NR][kFewRound];       // times the row's weight
    __shared__ __attribute__((aligned(32))) float fold[kFewThreads][E];
    const int tid = threadIdx.x;
    const int column = tid & (a.columns - 1), deal = tid / a.columns, deals = kFewThreads / a.columns;
    const int d = E * (blockIdx.y * a.columns + column), left = a.D - d;
    const T* const w = (const T*)a.w;
    vef x[NR], dx[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const vef u = widen(raw_of<E>((const T*)a.x + n * a.x_pitch, d, a.D));
        x[n] = a.weight[n] != 0.f ? u : vef{};
        dx[n] = vef{};
    }
    const long begin = (long)blockIdx.x * a.each, end = begin + a.each < a.V ? begin + a.each : a.V;
    for (long v0 = begin; v0 < end; v0 += kFewRound) {
        const int count = end - v0 < kFewRound ? (int)(end - v0) : kFewRound;
        for (int i = tid; i < NR * kFewRound; i += kFewThreads) {
            const int k = i / NR, n = i % NR;
            float g = 0.f;
            if (k < count) {
                const float weight = a.weight[n], s = a.scores[(v0 + k) * a.score_row + n];
                if (weight != 0.f) {
                    g = s == -__builtin_inff() ? 0.f : expf(s - a.lse[n]);
                    if (v0 + k == a.mask.labels[n]) g -= 1.f;
                    g *= weight;
                }
            }
            delta[n][k] = g;
        }
        __syncthreads();
        if (a.db && blockIdx.y == 0 && tid < count) {
            float s = 0.f;
#pragma unroll
            for (int n = 0; n < NR; ++n) s += delta[n][tid];
            a.db[v0 + tid] = s;
        }
        if (left > 0) {
            constexpr int U = 8;                 // classes in flight
            for (int k0 = deal; k0 < count; k0 += U * deals) {
                Raw<T, E> u[U];
#pragma unroll
                    for (int q = 0; q < U; ++q) {
                        const int k = k0 + q * deals;
                        u[q] = raw_of<E>(w + (v0 + (k < count ? k : count - 1)) * a.w_pitch, d, a.D);
                    }
#pragma unroll
                for (int q = 0; q < U; ++q) {
                    const int k = k0 + q * deals;
                    if (k >= count) break;
                    vef dw = {};
                    const vef v = widen(u[q]);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        const float g = delta[n][k];
#pragma unroll
                            for (int z = 0; z < E; ++z) dx[n][z] = fmaf(g, v[z], dx[n][z]);
#pragma unroll
                        for (int z = 0; z < E; ++z) dw[z] = fmaf(g, x[n][z], dw[z]);
                    }
                    if (a.dw) {
                        T* const to = (T*)a.dw + (v0 + k) * a.D + d;
                        if (left >= E) {
                            store_any(to, dw);
                        } else {
#pragma unroll
                            for (int z = 0; z < E; ++z)
                                if (z < left) store1(to + z, dw[z]);
                        }
                    }
                }
            }
        }
        __syncthreads();
    }
    if (!a.part) return;
#pragma unroll
    for (int n = 0; n < NR; ++n) {               // the deals of a class's features, in their order
        *reinterpret_cast<vef*>(fold[tid]) = dx[n];
        __syncthreads();
        if (deal == 0 && left > 0) {
            vef s = dx[n];
            for (int q = 1; q < deals; ++q) {
                const vef o = *reinterpret_cast<const vef*>(fold[q * a.columns + column]);
#pragma unroll
                for (int z = 0; z < E; ++z) s[z] += o[z];
            }
            float* const to = a.part + ((long)blockIdx.x * a.N + n) * a.D + d;
#pragma unroll
            for (int z = 0; z < E; ++z)
                if (z < left) to[z] = s[z];
        }
        __syncthreads();
    }
}

// dx from the shares: 64 numbers per workgroup, the shares dealt to 16 waves
template <typename T>
__global__ __launch_bounds__(1024) void rows_few_sum_kernel(FewArgs a)
{
    __shared__ double red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (blockIdx.x == 0 && a.loss && wave == 0) {
        double s = 0.0;
        for (int i = lane; i < a.loss_parts; i += 64) s += a.loss_part[i];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
        if (lane == 0) *a.loss = s;
    }
    const long all = (long)a.N * a.D, e = (long)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (a.part && e < all) {
        int p = wave;
        for (; p + 7 * 16 < a.parts; p += 8 * 16) {      // eight loads in flight
            float v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = a.part[(p + 16 * q) * all + e];
#pragma unroll
            for (int q = 0; q < 8; ++q) s += (double)v[q];
        }
        for (; p < a.parts; p += 16) s += (double)a.part[p * all + e];
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || !a.part || e >= all) return;
    for (int w = 1; w < 16; ++w) s += red[w][lane];
    const int n = (int)(e / a.D), d = (int)(e - (long)n * a.D);
    store1((T*)a.dx + n * a.dx_pitch + d, a.weight[n] == 0.f ? 0.f : (float)s);
}

}  // namespace mpcnn
