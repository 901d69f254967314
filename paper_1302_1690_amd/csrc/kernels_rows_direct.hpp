// The class layer on rows of features in few launches, for little work (class_rows.hip): the products read features, class weights and scores
// where they are, at any pitch and address, without being brought into blocks first, and without a stop in LDS.
//
//   rows_direct_scores   scores with their bias, stored [class][row], and per row and tile of classes the largest and the sum of exponentials
//   (rows_join_kernel    joins them; kernels_rows_parts.hpp)
//   rows_direct_grads    tiles of dx and of dw: the derivative is made from the scores on the way into the product.  A long sum is split over
//                        workgroups, which leave partial sums, and
//   rows_direct_sum      adds them up in their order.
//
// Products on v_mfma_f32_32x32x16_bf16: bf16 numbers as they are, fp32 ones as three bf16 parts (x = h + m + l, 24 bits) and the six largest
// of nine products: the same exponents as fp32, so no scale has to be found first, which is what two fp16 parts need and what costs
// two more passes.  A lane fetches its own operand, 8 k's of one row, a step (32 k's) ahead of the products; operands are fetched by every
// wave that needs them (first-level cache).  Little work is bound by the trips to memory one after the other, some 0.7 us each, and
// so a workgroup has one tile of 32 x 32 and its four waves deal the sum's steps among them; where there are tiles enough or the
// sum has a step or two, each wave has a tile of its own (64 x 64 per workgroup).
#pragma once
#include "any_address.hpp"
#include "kernels_rows_parts.hpp"

namespace mpcnn {

constexpr int kDirectK = 32;
constexpr float kLog2eHigh = 1.4426950408889634f, kLog2eLow = 1.925963033500212e-08f;   // log2 e in two fp32 numbers

typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 d_bf16x8 __attribute__((ext_vector_type(8)));

struct DirectArgs {
    const void *x, *w;
    long x_pitch, w_pitch;                 // elements
    int N, D, V;
    const float* bias;
    RowMask mask;
    float* scores;                         // [V][score_row], or null
    long score_row;
    float2* stats;                         // [tiles of classes][N]
    float* label_score;
    int score_deal, x_deal, w_deal;        // waves that deal a tile's sum among them: 4 (tiles of 32 x 32) or 1 (64 x 64)
    // gradients
    const float *lse, *weight;             // [Np], whole steps: weight 0 and
    const int* label;                      // label kNoLabel for rows that add nothing and behind the last
    void* dx;
    long dx_pitch;
    void* dw;
    float* db;
    int x_along, w_along;                  // tiles along the features
    int x_splits, x_each, w_splits, w_each;   // parts of the sums over classes and over rows, and their lengths (multiples of kDirectK)
    int x_groups, w_groups;                // workgroups of dx, of dw (0: not asked for)
    float *x_part, *w_part, *db_part;      // [split][N][D], [split][V][D], [split][V]: where splits > 1
    const double* loss_part;
    int loss_parts;
    double* loss;
};

template <typename T> constexpr int kDirectParts = sizeof(T) == 4 ? 3 : 1;

template <typename T>
__device__ __forceinline__ void direct_parts(d_bf16x8 (&p)[kDirectParts<T>], v8f v)
{
    p[0] = __builtin_convertvector(v, d_bf16x8);
    if constexpr (kDirectParts<T> == 3) {
        const v8f r = v - __builtin_convertvector(p[0], v8f);
        p[1] = __builtin_convertvector(r, d_bf16x8);
        p[2] = __builtin_convertvector(r - __builtin_convertvector(p[1], v8f), d_bf16x8);
    }
}
// acc += 16 k's
template <typename T>
__device__ __forceinline__ void direct_product(v16f& acc, v8f x, v8f y)
{
    constexpr int P = kDirectParts<T>;
    d_bf16x8 a[P], b[P];
    direct_parts<T>(a, x);
    direct_parts<T>(b, y);
#pragma unroll
    for (int sum = P - 1; sum >= 0; --sum)              // the smallest products first
#pragma unroll
        for (int i = 0; i <= sum; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[sum - i], acc, 0, 0, 0);
}

// The sums of the four waves' accumulators, in their order: thread t the results [4 (t / 32) + q][t % 32] of the tile
__device__ __forceinline__ v4f direct_fold(const v16f& acc, float (*fold)[32][33])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int r = 0; r < 16; ++r) fold[wave][8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)][lane & 31] = acc[r];
    __syncthreads();
    v4f s;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int m = 4 * (threadIdx.x >> 5) + q, n = threadIdx.x & 31;
        s[q] = ((fold[0][m][n] + fold[1][m][n]) + fold[2][m][n]) + fold[3][m][n];
    }
    return s;
}

__device__ __forceinline__ float2 direct_join(float2 s, float2 o)
{
    const float t = fmaxf(s.x, o.x), b = t == -__builtin_inff() ? 0.f : t;
    return float2{t, s.y * __expf(s.x - b) + o.y * __expf(o.x - b)};
}

template <typename T>
__global__ __launch_bounds__(256) void rows_direct_scores_kernel(DirectArgs a)
{
    __shared__ float fold[4][32][33];
    __shared__ float2 red[8][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool deal = a.score_deal == 4;                 // (uniform)
    const int side = deal ? 32 : 64;
    const int v0 = blockIdx.x * side + (deal ? 0 : 32 * (wave >> 1)), n0 = blockIdx.y * side + (deal ? 0 : 32 * (wave & 1));
    const int row = lane & 31, half = lane >> 5;
    const int va = v0 + row < a.V ? v0 + row : a.V - 1, nb = n0 + row < a.N ? n0 + row : a.N - 1;
    const T* const pa = (const T*)a.w + va * a.w_pitch;
    const T* const pb = (const T*)a.x + nb * a.x_pitch;
    v16f acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    const int steps = (a.D + kDirectK - 1) / kDirectK, whole = a.D / kDirectK, first = deal ? wave : 0, by = deal ? 4 : 1;
    Raw8<T> u[2], y[2];
    auto fetch = [&](int s) {
        if (s < whole) {
#pragma unroll
            for (int k = 0; k < 2; ++k) { u[k] = raw8(pa + kDirectK * s + 16 * k + 8 * half); y[k] = raw8(pb + kDirectK * s + 16 * k + 8 * half); }
        } else if (s < steps) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                u[k] = raw8_of(pa, kDirectK * s + 16 * k + 8 * half, a.D);
                y[k] = raw8_of(pb, kDirectK * s + 16 * k + 8 * half, a.D);
            }
        }
    };
    fetch(first);
    for (int s = first; s < steps; s += by) {
        const v8f a0 = widen(u[0]), a1 = widen(u[1]), b0 = widen(y[0]), b1 = widen(y[1]);
        fetch(s + by);
        direct_product<T>(acc, a0, b0);
        direct_product<T>(acc, a1, b1);
    }
    constexpr float kNone = -__builtin_inff();
    if (deal) {
        v4f s = direct_fold(acc, fold);
        const int n = n0 + (tid & 31), m0 = v0 + 4 * (tid >> 5);
        const bool real = n < a.N;
        const int label = real ? a.mask.labels[n] : -1;
        float top = kNone;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int m = m0 + q;
            const float b = a.bias ? a.bias[m < a.V ? m : a.V - 1] : 0.f;
            s[q] = m < a.V ? s[q] + b : kNone;
            top = fmaxf(top, s[q]);
            if (m < a.V && real) {
                if (a.scores) a.scores[m * a.score_row + n] = s[q];
                if (m == label) a.label_score[n] = s[q];
            }
        }
        const float base = top == kNone ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) sum += __expf(s[q] - base);
        red[tid >> 5][tid & 31] = float2{top, sum};
        __syncthreads();
        if (tid < 32 && n0 + tid < a.N) {
            float2 t = red[0][tid];
#pragma unroll
            for (int q = 1; q < 8; ++q) t = direct_join(t, red[q][tid]);
            a.stats[(long)blockIdx.x * a.N + n0 + tid] = t;
        }
        return;
    }
    const int m0 = v0 + 4 * half, n = n0 + row;
    const bool real = n < a.N;
    const int label = real ? a.mask.labels[n] : -1;
    float bias[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int m = m0 + 8 * (r >> 2) + (r & 3);
        bias[r] = a.bias ? a.bias[m < a.V ? m : a.V - 1] : 0.f;
    }
    float top = kNone;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int m = m0 + 8 * (r >> 2) + (r & 3);
        const float v = m < a.V ? acc[r] + bias[r] : kNone;
        acc[r] = v;
        top = fmaxf(top, v);
        if (m < a.V && real) {
            if (a.scores) a.scores[m * a.score_row + n] = v;
            if (m == label) a.label_score[n] = v;
        }
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float base = top == kNone ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += __expf(acc[r] - base);
    sum += __shfl_xor(sum, 32, 64);
    if (half == 0) red[wave >> 1][32 * (wave & 1) + row] = float2{top, sum};
    __syncthreads();
    const int nt = blockIdx.y * 64 + tid;
    if (tid < 64 && nt < a.N) a.stats[(long)blockIdx.x * a.N + nt] = direct_join(red[0][tid], red[1][tid]);
}

// exp(score - lse) - hot; nothing for rows that are not live.  exp by the hardware's exp2, whose argument's rounding is made good: x log2 e = t + r
// to twice fp32's bits, 2^(t + r) = 2^t (1 + r ln 2) for |r| below a 2^-24th of t.
__device__ __forceinline__ float direct_delta(float score, float lse, bool live, bool hot)
{
    const float x = score == -__builtin_inff() ? -1e30f : score - lse;     // (a class that is switched off, and a row that has no other)
    const float t = x * kLog2eHigh, r = fmaf(x, kLog2eHigh, -t) + x * kLog2eLow;
    const float e = __builtin_amdgcn_exp2f(t);
    const float p = e > 0.f ? fmaf(e, r * 0.6931471805599453f, e) : e;
    return live ? (hot ? p - 1.f : p) : 0.f;
}

template <typename T>
__global__ __launch_bounds__(256) void rows_direct_grads_kernel(DirectArgs a)
{
    __shared__ float fold[4][32][33];
    __shared__ double red[256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = lane & 31, half = lane >> 5;
    int id = blockIdx.x;
    if (id == 0 && a.loss) {                             // the summed loss, in a fixed order
        double s = 0.0;
        for (int i = tid; i < a.loss_parts; i += 256) s += a.loss_part[i];
        red[tid] = s;
        __syncthreads();
        for (int w = 128; w > 0; w >>= 1) {
            if (tid < w) red[tid] += red[tid + w];
            __syncthreads();
        }
        if (tid == 0) *a.loss = red[0];
    }
    const bool dx = id < a.x_groups;
    if (!dx) id -= a.x_groups;
    if (!dx && id >= a.w_groups) return;                 // (a launch for the loss alone)
    const bool deal = (dx ? a.x_deal : a.w_deal) == 4;
    const int splits = dx ? a.x_splits : a.w_splits, each = dx ? a.x_each : a.w_each, along = dx ? a.x_along : a.w_along;
    const int K = dx ? a.V : a.N, M = dx ? a.N : a.V;
    const int tile = id / splits, split = id - tile * splits;
    const int mt = tile / along, dt = tile - mt * along;
    const int side = deal ? 32 : 64;
    const int m0 = mt * side + (deal ? 0 : 32 * (wave >> 1)), d0 = dt * side + (deal ? 0 : 32 * (wave & 1)), k0 = split * each;
    const int len = K - k0 < each ? K - k0 : each, steps = (len + kDirectK - 1) / kDirectK;
    const int first = deal ? wave : 0, by = deal ? 4 : 1;
    v16f acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    const int d = d0 + row < a.D ? d0 + row : a.D - 1;
    const int m = m0 + row < M ? m0 + row : M - 1;
    float bias = 0.f;
    if (dx) {
        const float lse = a.lse[m];
        const int label = a.label[m];
        const T* const w = (const T*)a.w + d;
        const float* const sc = a.scores + m;
        float u[16];
        T y[16];
        auto fetch = [&](int s) {                        // scores [class][row], weights [class][feature]: lanes side by side, 8 k's one below the other
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int v = k0 + s * kDirectK + 16 * (z >> 3) + 8 * half + (z & 7), at = v < a.V ? v : a.V - 1;
                u[z] = sc[at * a.score_row];
                y[z] = w[at * a.w_pitch];
            }
        };
        if (first < steps) fetch(first);
        for (int s = first; s < steps; s += by) {
            v8f p[2], q[2];
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int v = k0 + s * kDirectK + 16 * (z >> 3) + 8 * half + (z & 7);
                p[z >> 3][z & 7] = direct_delta(u[z], lse, label != kNoLabel && v < a.V, v == label);
                q[z >> 3][z & 7] = (float)y[z];          // (beyond the last class times a derivative of zero: finite or not finite anyway)
            }
            if (s + by < steps) fetch(s + by);
            direct_product<T>(acc, p[0], q[0]);
            direct_product<T>(acc, p[1], q[1]);
        }
    } else {
        const float* const sc = a.scores + m * a.score_row;
        const T* const x = (const T*)a.x + d;
        v8f u[2], l[2], w8[2];
        v4i t[4];
        T y[16];
        auto fetch = [&](int s) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int n = k0 + s * kDirectK + 16 * k + 8 * half;    // (scores, lse, weight and label are padded to whole steps)
                u[k] = load8(sc + n);
                l[k] = load8(a.lse + n);
                w8[k] = load8(a.weight + n);
                t[2 * k] = *reinterpret_cast<const v4i*>(a.label + n);
                t[2 * k + 1] = *reinterpret_cast<const v4i*>(a.label + n + 4);
            }
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int n = k0 + s * kDirectK + 16 * (z >> 3) + 8 * half + (z & 7);
                y[z] = x[(n < a.N ? n : a.N - 1) * a.x_pitch];
            }
        };
        if (first < steps) fetch(first);
        for (int s = first; s < steps; s += by) {
            v8f p[2], q[2];
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int k = z >> 3, label = t[z >> 2][z & 3];
                const bool live = label != kNoLabel;
                const float g = direct_delta(u[k][z & 7], l[k][z & 7], live, label == m) * w8[k][z & 7];
                p[k][z & 7] = g;
                bias += g;
                q[k][z & 7] = live ? (float)y[z] : 0.f;
            }
            if (s + by < steps) fetch(s + by);
            direct_product<T>(acc, p[0], q[0]);
            direct_product<T>(acc, p[1], q[1]);
        }
        bias += __shfl_xor(bias, 32, 64);
    }

    const bool whole = splits == 1;
    auto put = [&](int m, int d, float v) {
        if (m >= M || d >= a.D) return;
        if (!whole) {
            (dx ? a.x_part : a.w_part)[((long)split * M + m) * a.D + d] = v;
        } else if (dx) {
            const float scale = a.weight[m];
            store1((T*)a.dx + m * a.dx_pitch + d, scale == 0.f ? 0.f : v * scale);
        } else if (a.dw) {
            store1((T*)a.dw + (long)m * a.D + d, v);
        }
    };
    float* const to_db = whole ? a.db : a.db_part + (long)split * a.V;
    if (deal) {
        const v4f s = direct_fold(acc, fold);
#pragma unroll
        for (int q = 0; q < 4; ++q) put(m0 + 4 * (tid >> 5) + q, d0 + (tid & 31), s[q]);
        if (!dx && dt == 0 && a.db) {
            __syncthreads();
            if (half == 0) fold[wave][0][row] = bias;
            __syncthreads();
            if (tid < 32 && m0 + tid < a.V) to_db[m0 + tid] = ((fold[0][0][tid] + fold[1][0][tid]) + fold[2][0][tid]) + fold[3][0][tid];
        }
        return;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) put(m0 + 8 * (r >> 2) + 4 * half + (r & 3), d0 + row, acc[r]);
    if (!dx && dt == 0 && a.db && (wave & 1) == 0 && half == 0 && m0 + row < a.V) to_db[m0 + row] = bias;
}

template <typename T>
__global__ __launch_bounds__(256) void rows_direct_sum_kernel(DirectArgs a)
{
    const long nx = a.x_part ? (long)a.N * a.D : 0, nw = a.w_part && a.dw ? (long)a.V * a.D : 0, nb = a.db_part && a.db ? a.V : 0;
    for (long e = (long)blockIdx.x * 256 + threadIdx.x; e < nx + nw + nb; e += (long)gridDim.x * 256) {
        const bool of_x = e < nx, of_w = !of_x && e < nx + nw;
        const long at = of_x ? e : of_w ? e - nx : e - nx - nw, by = of_x ? nx : of_w ? (long)a.V * a.D : a.V;
        const float* const part = (of_x ? a.x_part : of_w ? a.w_part : a.db_part) + at;
        const int splits = of_x ? a.x_splits : a.w_splits;
        float s = 0.f;
        int i = 0;
        for (; i + 7 < splits; i += 8) {                 // eight loads in flight
            float v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = part[(i + q) * by];
#pragma unroll
            for (int q = 0; q < 8; ++q) s += v[q];
        }
        for (; i < splits; ++i) s += part[i * by];
        if (of_x) {
            const long n = at / a.D;
            const float scale = a.weight[n];
            store1((T*)a.dx + n * a.dx_pitch + (at - n * a.D), scale == 0.f ? 0.f : s * scale);
        } else if (of_w) {
            store1((T*)a.dw + at, s);
        } else {
            a.db[at] = s;
        }
    }
}

}  // namespace mpcnn
