// The class layer on rows of features in three launches, for few rows or little work (class_rows.hip): the products read features, class
// weights and scores where they are, at any pitch and address, without being brought into blocks first.
//
//   rows_direct_scores   a tile of 64 classes x 64 rows: scores with their bias, stored [class][row], and per row the tile's largest and sum
//                        of exponentials
//   (rows_join_kernel    joins them; kernels_rows_parts.hpp)
//   rows_direct_grads    tiles of 64 rows x 64 features of dx and of 64 classes x 64 features of dw: the derivative is made from the scores
//                        on the way into the product.  A long sum is split over workgroups; the one of a tile that ends last adds up their
//                        partial sums, in their order, so that the result does not depend on which one that is.
//
// Products on v_mfma_f32_32x32x16_bf16: bf16 numbers as they are, fp32 ones as three bf16 parts (x = h + m + l, 24 bits) and the six largest
// of nine products: the same exponents as fp32, so no scale has to be found first, which is what two fp16 parts need and what costs
// two more passes.  A thread fetches 8 k's of one row per step of 32 k's, one step ahead of the products, and leaves them in LDS as
// 128-bit words per part; rows of 64 bytes per part and 16 more, which puts 16 lanes' fetches on different banks.
//
// Bound by latency where the work is little (a workgroup per compute unit or less, some 32 k's per microsecond each), by the passes over the
// class weights (twice read, their gradient written) where the rows are few.
#pragma once
#include "any_address.hpp"
#include "kernels_rows_parts.hpp"

namespace mpcnn {

constexpr int kDirectSide = 64, kDirectK = 32;
constexpr float kLog2eHigh = 1.4426950408889634f, kLog2eLow = 1.925963033500212e-08f;   // log2 e in two fp32 numbers

typedef __bf16 d_bf16x8 __attribute__((ext_vector_type(8)));

struct DirectArgs {
    const void *x, *w;
    long x_pitch, w_pitch;                 // elements
    int N, D, V;
    const float* bias;
    RowMask mask;
    float* scores;                         // [V][score_row]; rows beyond the last are not read as such
    long score_row;
    float2* stats;                         // [tiles of classes][N]
    float* label_score;
    int store;
    // gradients
    const float *lse, *weight;             // [Np], whole steps: weight 0 and
    const int* label;                      // label kNoLabel for rows that add nothing and behind the last
    void* dx;
    long dx_pitch;
    void* dw;
    float* db;
    int x_tiles, w_tiles, d_tiles;         // tiles of rows, of classes, of features
    int x_splits, x_each, w_splits, w_each;   // parts of the sums over classes and over rows, and their lengths (multiples of kDirectK)
    int x_groups, w_groups;                // workgroups of dx, of dw (0: not asked for)
    float *x_part, *w_part, *db_part;      // [tile][split][64][64], [class tile][split][64]
    unsigned* tickets;                     // per tile; zero
    const double* loss_part;
    int loss_parts;
    double* loss;
};

template <typename T> constexpr int kDirectParts = sizeof(T) == 4 ? 3 : 1;
template <typename T> constexpr int kDirectPitch = kDirectParts<T> * 64 + 16;
template <typename T> constexpr int kDirectStage = kDirectSide * kDirectPitch<T>;   // bytes of one operand

// 8 numbers of a thread's row into its LDS place
template <typename T>
__device__ __forceinline__ void direct_put(char* at, v8f v)
{
    const d_bf16x8 h = __builtin_convertvector(v, d_bf16x8);
    *reinterpret_cast<d_bf16x8*>(at) = h;
    if constexpr (kDirectParts<T> == 3) {
        const v8f r = v - __builtin_convertvector(h, v8f);
        const d_bf16x8 m = __builtin_convertvector(r, d_bf16x8);
        *reinterpret_cast<d_bf16x8*>(at + 64) = m;
        *reinterpret_cast<d_bf16x8*>(at + 128) = __builtin_convertvector(r - __builtin_convertvector(m, v8f), d_bf16x8);
    }
}

// acc += A B over `steps` steps of 32 k's.  fetch_a(step), fetch_b(step) give the thread's 8 numbers of a step; at_a, at_b: their places.
template <typename T, typename FA, typename FB>
__device__ __forceinline__ void direct_product(v16f& acc, char* lds, int steps, int at_a, int at_b, FA fetch_a, FB fetch_b)
{
    constexpr int P = kDirectParts<T>, pitch = kDirectPitch<T>, stage = kDirectStage<T>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int of_a = (32 * (wave >> 1) + (lane & 31)) * pitch + 16 * (lane >> 5);
    const int of_b = stage + (32 * (wave & 1) + (lane & 31)) * pitch + 16 * (lane >> 5);
    if (steps <= 0) return;
    v8f va = fetch_a(0), vb = fetch_b(0);
    for (int s = 0; s < steps; ++s) {
        char* buf = lds + (s & 1) * 2 * stage;
        direct_put<T>(buf + at_a, va);
        direct_put<T>(buf + stage + at_b, vb);
        if (s + 1 < steps) { va = fetch_a(s + 1); vb = fetch_b(s + 1); }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            d_bf16x8 a[P], b[P];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                a[p] = *reinterpret_cast<const d_bf16x8*>(buf + of_a + 64 * p + 32 * k);
                b[p] = *reinterpret_cast<const d_bf16x8*>(buf + of_b + 64 * p + 32 * k);
            }
#pragma unroll
            for (int sum = P - 1; sum >= 0; --sum)      // the smallest products first
#pragma unroll
                for (int i = 0; i <= sum; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[sum - i], acc, 0, 0, 0);
        }
    }
    __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(256) void rows_direct_scores_kernel(DirectArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[4 * kDirectStage<T>];
    __shared__ float2 red[2][kDirectSide];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int v0 = blockIdx.x * kDirectSide, n0 = blockIdx.y * kDirectSide;
    const int row = tid >> 2, oct = tid & 3;             // fetches: a row's 8 k's, four threads a row
    const int va = v0 + row < a.V ? v0 + row : a.V - 1, nb = n0 + row < a.N ? n0 + row : a.N - 1;
    const T* const pa = (const T*)a.w + va * a.w_pitch;
    const T* const pb = (const T*)a.x + nb * a.x_pitch;
    v16f acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    const int at = row * kDirectPitch<T> + 16 * oct;
    direct_product<T>(acc, lds, (a.D + kDirectK - 1) / kDirectK, at, at,
                      [&](int s) { return load8_of(pa, s * kDirectK + 8 * oct, a.D); },
                      [&](int s) { return load8_of(pb, s * kDirectK + 8 * oct, a.D); });
    constexpr float kNone = -__builtin_inff();
    const int half = lane >> 5, m0 = v0 + 32 * (wave >> 1) + 4 * half, n = n0 + 32 * (wave & 1) + (lane & 31);
    const bool real = n < a.N;
    const int label = real ? a.mask.labels[n] : -1;
    float top = kNone;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int m = m0 + 8 * (r >> 2) + (r & 3);
        const float v = m < a.V ? acc[r] + (a.bias ? a.bias[m] : 0.f) : kNone;
        acc[r] = v;
        top = fmaxf(top, v);
        if (m < a.V && real) {
            if (a.store) a.scores[m * a.score_row + n] = v;
            if (m == label) a.label_score[n] = v;
        }
    }
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float base = top == kNone ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += __expf(acc[r] - base);
    sum += __shfl_xor(sum, 32, 64);
    if (half == 0) red[wave >> 1][32 * (wave & 1) + (lane & 31)] = float2{top, sum};
    __syncthreads();
    if (tid < kDirectSide && n0 + tid < a.N) {
        const float2 s = red[0][tid], o = red[1][tid];
        const float t = fmaxf(s.x, o.x), b = t == kNone ? 0.f : t;
        a.stats[(long)blockIdx.x * a.N + n0 + tid] = float2{t, s.y * __expf(s.x - b) + o.y * __expf(o.x - b)};
    }
}

// exp(score - lse) - hot, nothing for rows of label kNoLabel.  exp by the hardware's exp2, whose argument's rounding is made good: x log2 e = t + r
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
    __shared__ __attribute__((aligned(16))) char lds[4 * kDirectStage<T>];
    __shared__ double red[256];
    __shared__ unsigned turn;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int half = lane >> 5;
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
    const int splits = dx ? a.x_splits : a.w_splits, each = dx ? a.x_each : a.w_each;
    const int K = dx ? a.V : a.N, M = dx ? a.N : a.V;
    if (!dx && id >= a.w_groups) return;                 // (a launch for the loss alone)
    const int tile = id / splits, split = id - tile * splits;
    const int mt = tile / a.d_tiles, dt = tile - mt * a.d_tiles;
    const int m0 = mt * kDirectSide, d0 = dt * kDirectSide, k0 = split * each;
    const int len = K - k0 < each ? K - k0 : each, steps = (len + kDirectK - 1) / kDirectK;

    v16f acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    const int across = lane, oct_c = __builtin_amdgcn_readfirstlane(wave);   // fetches along the rows of memory: lanes side by side, 8 k's one below the other
    const int at_c = across * kDirectPitch<T> + 16 * oct_c;
    const int d = d0 + across < a.D ? d0 + across : a.D - 1;
    float bias = 0.f;
    if (dx) {
        const int n = m0 + across < a.N ? m0 + across : a.N - 1;
        const float lse = a.lse[n];
        const int label = a.label[n];
        const T* const w = (const T*)a.w + d;
        const float* const sc = a.scores + n;
        direct_product<T>(acc, lds, steps, at_c, at_c,
                          [&](int s) {
                              const int v = k0 + s * kDirectK + 8 * oct_c;
                              float x[8];
                              v8f r;
#pragma unroll
                              for (int z = 0; z < 8; ++z) x[z] = sc[(v + z < a.V ? v + z : a.V - 1) * a.score_row];
#pragma unroll
                              for (int z = 0; z < 8; ++z) r[z] = direct_delta(x[z], lse, label != kNoLabel && v + z < a.V, v + z == label);
                              return r;
                          },
                          [&](int s) {
                              const int v = k0 + s * kDirectK + 8 * oct_c;
                              v8f r;
#pragma unroll
                              for (int z = 0; z < 8; ++z) r[z] = load1(w + (v + z < a.V ? v + z : a.V - 1) * a.w_pitch);
                              return r;                  // (beyond the last class times a derivative of zero: finite or not finite anyway)
                          });
    } else {
        const int row = tid >> 2, oct = tid & 3;
        const int v = m0 + row < a.V ? m0 + row : a.V - 1;
        const float* const sc = a.scores + v * a.score_row + 8 * oct;
        const bool sums = dt == 0 && a.db;
        const T* const x = (const T*)a.x + d;
        direct_product<T>(acc, lds, steps, row * kDirectPitch<T> + 16 * oct, at_c,
                          [&](int s) {
                              const int n = k0 + s * kDirectK;
                              const v8f x8 = load8(sc + n), l8 = load8(a.lse + n + 8 * oct), w8 = load8(a.weight + n + 8 * oct);
                              const v4f t0 = load4((const float*)a.label + n + 8 * oct), t1 = load4((const float*)a.label + n + 8 * oct + 4);
                              v8f r;
#pragma unroll
                              for (int z = 0; z < 8; ++z) {
                                  const int label = __builtin_bit_cast(int, z < 4 ? t0[z & 3] : t1[z & 3]);
                                  r[z] = direct_delta(x8[z], l8[z], label != kNoLabel, label == v) * w8[z];
                                  bias += r[z];
                              }
                              return r;
                          },
                          [&](int s) {
                              const int n = k0 + s * kDirectK + 8 * oct_c;
                              float u[8];
                              v8f r;
#pragma unroll
                              for (int z = 0; z < 8; ++z) u[z] = load1(x + (n + z < a.N ? n + z : a.N - 1) * a.x_pitch);
#pragma unroll
                              for (int z = 0; z < 8; ++z) r[z] = a.label[n + z] != kNoLabel ? u[z] : 0.f;
                              return r;
                          });
        bias = sums ? bias : 0.f;
        bias += __shfl_xor(bias, 1, 64);
        bias += __shfl_xor(bias, 2, 64);
    }

    // ---- whole sums, or partial ones and whoever comes last adds them up
    const int mw = 32 * (wave >> 1) + 4 * half, dw_ = 32 * (wave & 1) + (lane & 31);
    const bool last_row = !dx && dt == 0 && a.db && (tid & 3) == 0;
    if (splits > 1) {
        float* const slots = (dx ? a.x_part : a.w_part) + (long)tile * splits * (kDirectSide * kDirectSide);
        float* const mine = slots + (long)split * (kDirectSide * kDirectSide);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int m = mw + 8 * (r >> 2) + (r & 3);
            if (m0 + m < M) mine[m * kDirectSide + dw_] = acc[r];
        }
        if (last_row) a.db_part[((long)mt * splits + split) * kDirectSide + (tid >> 2)] = bias;
        __threadfence();
        __syncthreads();
        if (tid == 0) turn = __hip_atomic_fetch_add(a.tickets + (dx ? 0 : a.x_tiles * a.d_tiles) + tile, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (turn != (unsigned)splits - 1) return;
        __threadfence();
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.f;
        for (int s = 0; s < splits; ++s) {
            float v[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int m = mw + 8 * (r >> 2) + (r & 3);
                v[r] = m0 + m < M ? slots[(long)s * (kDirectSide * kDirectSide) + m * kDirectSide + dw_] : 0.f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] += v[r];
        }
        if (last_row) {
            bias = 0.f;
            for (int s = 0; s < splits; ++s) bias += a.db_part[((long)mt * splits + s) * kDirectSide + (tid >> 2)];
        }
    }
    if (last_row && m0 + (tid >> 2) < a.V) a.db[m0 + (tid >> 2)] = bias;
    if (d0 + dw_ >= a.D) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int m = m0 + mw + 8 * (r >> 2) + (r & 3);
        if (m >= M) continue;
        if (dx) {
            const float scale = a.weight[m];
            store1((T*)a.dx + m * a.dx_pitch + d0 + dw_, scale == 0.f ? 0.f : acc[r] * scale);
        } else {
            if (a.dw) store1((T*)a.dw + (long)m * a.D + d0 + dw_, acc[r]);
        }
    }
}

}  // namespace mpcnn
