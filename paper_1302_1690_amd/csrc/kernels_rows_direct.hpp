// The class layer on rows of features in few launches, for little work (class_rows.hip): the products read features, class weights and scores
// where they are, at any pitch and address, without being brought into blocks first, and without a stop in LDS.
//
//   rows_direct_scores   scores with their bias, stored [class][row], and per row and tile of classes the largest and the sum of exponentials
//   rows_direct_delta    joins them (where there are few tiles; else rows_join_kernel has) and turns the scores into the loss's derivative times
//                        the row's weight: made once, not by every tile of features (20 instructions each, which bound the gradients)
//   rows_direct_grads    tiles of dx and of dw, and the bias gradients' sums.  A long sum is split over workgroups, which leave partial sums, and
//   rows_direct_sum      adds them up in their order (where there are any).
//
// Products on v_mfma_f32_32x32x16_bf16: bf16 numbers as they are, fp32 ones as three bf16 parts (x = h + m + l, 24 bits) and the six largest
// of nine products: the same exponents as fp32, so no scale has to be found first, which is what two fp16 parts need and what costs
// two more passes.  The derivative stays fp32 with either storage; for bf16 storage it is multiplied as two parts (16 bits), so that results
// are rounded once.  A lane fetches its own operand, 8 k's of one row, a step (32 k's) ahead of the products; operands are fetched by every
// wave that needs them (first-level cache).  Little work is bound by the trips to memory one after the other, some 0.7 us each, and
// so a workgroup has one tile of 32 x 32 and its four waves deal the sum's steps among them; where there are tiles enough or the
// sum has a step or two, each wave has a tile of its own (64 x 64 per workgroup).  213 x 100 x 37 fp32: 7.0 + 6.7 + 6.3 us.
#pragma once
#include "any_address.hpp"
#include "kernels_rows_parts.hpp"

namespace mpcnn {

constexpr int kDirectK = 32;

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
    const char* x_split;                   // features as operands (rows_split_kernel)
    int x_tiles;                           // of 32 rows, a multiple of the kernel's
    int score_deal, x_deal, w_deal;        // waves that deal a tile's sum among them: 4 (tiles of 32 x 32) or 1 (64 x 64)
    // derivative
    float *lse, *weight;                   // [N]; lse null: joined here
    float *rowloss, *lse_out;              // results of the join (null: not asked for)
    int tiles, batch;                      // of the statistics; of the derivative: times 64 rows per workgroup
    double* shares;                        // of the loss, one per workgroup along the rows, or null
    int delta;                             // whether the derivative takes the scores' place, zeros for rows that add nothing
    // gradients
    void* dx;
    long dx_pitch;
    void* dw;
    float* db;
    int x_along, w_along;                  // tiles along the features
    int x_splits, x_each, w_splits, w_each;   // parts of the sums over classes and over rows, and their lengths (multiples of kDirectK)
    int x_groups, w_groups;                // workgroups of dx, of dw (0: not asked for)
    float *x_part, *w_part;                // [split][N][D], [split][V][D]: where splits > 1
    float* db_part;                        // [db_parts][V]: where the derivative's rows are taken by several workgroups
    int db_parts, db_groups;               // and the workgroups that add them up
    const double* loss_part;
    int loss_parts;
    double* loss;
};

template <int P>
__device__ __forceinline__ void direct_parts(d_bf16x8 (&p)[P], v8f v)
{
    p[0] = __builtin_convertvector(v, d_bf16x8);
    if constexpr (P > 1) {
        const v8f r = v - __builtin_convertvector(p[0], v8f);
        p[1] = __builtin_convertvector(r, d_bf16x8);
        if constexpr (P > 2) p[2] = __builtin_convertvector(r - __builtin_convertvector(p[1], v8f), d_bf16x8);
    }
}
// acc += 16 k's, x in PA parts, y in PB
template <int PA, int PB>
__device__ __forceinline__ void direct_product(v16f& acc, v8f x, v8f y)
{
    constexpr int P = PA > PB ? PA : PB;
    d_bf16x8 a[PA], b[PB];
    direct_parts<PA>(a, x);
    direct_parts<PB>(b, y);
#pragma unroll
    for (int sum = P - 1; sum >= 0; --sum)              // the smallest products first
#pragma unroll
        for (int i = 0; i <= sum; ++i)
            if (i < PA && sum - i < PB) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b[sum - i], acc, 0, 0, 0);
}
template <typename T> constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
template <typename T> constexpr int kDeltaParts = sizeof(T) == 4 ? 3 : 2;

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

// ODD: of bf16 rows some begin at addresses that are no multiple of four (any_address.hpp).  The loss of 23 x 2541 x 10715: 48 us without, 30 with it;
// of 23 x 2544 x 10715: 18 us.
template <typename T, bool ODD>
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
    std::conditional_t<ODD, Odd8, Raw8<T>> u[2], y[2];
    auto fetch = [&](int s) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = kDirectK * s + 16 * k + 8 * half;
            if (s < whole) {
                if constexpr (ODD) { u[k] = odd8(pa + at); y[k] = odd8(pb + at); }
                else { u[k] = raw8(pa + at); y[k] = raw8(pb + at); }
            } else if (s < steps) {
                if constexpr (ODD) { u[k] = odd8_of(pa, at, a.D); y[k] = odd8_of(pb, at, a.D); }
                else { u[k] = raw8_of(pa, at, a.D); y[k] = raw8_of(pb, at, a.D); }
            }
        }
    };
    auto wide = [&](const auto& v, const T* row) { if constexpr (ODD) return widen(v, row); else return widen(v); };   // (steps are whole words)
    fetch(first);
    for (int s = first; s < steps; s += by) {
        const v8f a0 = wide(u[0], pa), a1 = wide(u[1], pa), b0 = wide(y[0], pb), b1 = wide(y[1], pb);
        fetch(s + by);
        direct_product<kParts<T>, kParts<T>>(acc, a0, b0);
        direct_product<kParts<T>, kParts<T>>(acc, a1, b1);
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

// ---- fp32 scores of some tens of rows over many classes: bound by the pass over the class weights, which a wave takes from memory into its operands
// and splits once for up to 64 rows.  The features are split before (rows_split_kernel), into operands as the lanes want them: [step of 32 k's][16 k's][part]
// [tile of 32 rows][lane], and come from the second-level cache, for 64 rows three times the class
// weights' bytes.  The waves deal the sum's steps among them.  64 x 4096 x 50000: a call of the loss 310 us, 2.6 TB/s of weights.  (Two steps of weights ahead: 8 % slower; two
// waves of other classes beside each other, which read the same features: 8 % slower.)
struct SplitArgs {
    const float* x;
    long x_pitch;
    int N, D, tiles;                       // of 32 rows
    char* out;
};
__global__ __launch_bounds__(256) void rows_split_kernel(SplitArgs a)
{
    const long all = (long)(a.D + kDirectK - 1) / kDirectK * 2 * a.tiles * 64;
    for (long e = (long)blockIdx.x * 256 + threadIdx.x; e < all; e += (long)gridDim.x * 256) {
        const int lane = (int)(e & 63), tile = (int)((e >> 6) % a.tiles);
        const long k16 = (e >> 6) / a.tiles;
        const int n = 32 * tile + (lane & 31);
        const v8f v = load8_of(a.x + (long)(n < a.N ? n : a.N - 1) * a.x_pitch, (int)(16 * k16) + 8 * (lane >> 5), a.D);
        d_bf16x8 p[3];
        direct_parts<3>(p, v);
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<d_bf16x8*>(a.out + (((k16 * 3 + i) * a.tiles + tile) * 64 + lane) * 16) = p[i];
    }
}
template <int NT>                          // tiles of 32 rows of a wave: 1 or 2
__global__ __launch_bounds__(256) void rows_wide_scores_kernel(DirectArgs a)
{
    constexpr float kNone = -__builtin_inff();
    __shared__ float fold[4][32][33];
    __shared__ float2 red[8][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int groups_n = a.x_tiles / NT;                 // (side by side: they read the same class weights)
    const int vt = blockIdx.x / groups_n, t0 = NT * (blockIdx.x - vt * groups_n), v0 = 32 * vt;
    const int row = lane & 31, half = lane >> 5;
    const float* const pw = (const float*)a.w + (long)(v0 + row < a.V ? v0 + row : a.V - 1) * a.w_pitch;
    const int steps = (a.D + kDirectK - 1) / kDirectK, whole = a.D / kDirectK;
    v16f acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[j][r] = 0.f;
    Raw8<float> u[2];
    d_bf16x8 x[2][3][NT];
    auto fetch_w = [&](int s) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int at = kDirectK * s + 16 * k + 8 * half;
            if (s < whole) u[k] = raw8(pw + at);
            else if (s < steps) u[k] = raw8_of(pw, at, a.D);
        }
    };
    auto fetch_x = [&](int s) {
        if (s >= steps) return;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 3; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    x[k][i][j] = *reinterpret_cast<const d_bf16x8*>(a.x_split + (((long)(2 * s + k) * 3 + i) * a.x_tiles + t0 + j) * 1024 + 16 * lane);
    };
    fetch_w(wave);
    fetch_x(wave);
    for (int s = wave; s < steps; s += 4) {
        d_bf16x8 w[2][3];
#pragma unroll
        for (int k = 0; k < 2; ++k) direct_parts<3>(w[k], widen(u[k]));
        fetch_w(s + 4);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int sum = 2; sum >= 0; --sum)       // the smallest products first
#pragma unroll
                    for (int i = 0; i <= sum; ++i) acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[k][i], x[k][sum - i][j], acc[j], 0, 0, 0);
        fetch_x(s + 4);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        v4f s = direct_fold(acc[j], fold);
        const int n0 = 32 * (t0 + j), n = n0 + (tid & 31), m0 = v0 + 4 * (tid >> 5);
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
        __syncthreads();                                 // (and the fold has been read)
        if (tid < 32 && n0 + tid < a.N) {
            float2 t = red[0][tid];
#pragma unroll
            for (int q = 1; q < 8; ++q) t = direct_join(t, red[q][tid]);
            a.stats[(long)vt * a.N + n0 + tid] = t;
        }
        __syncthreads();
    }
}

// 64 classes x `batch` times 64 rows per workgroup: a lane a row, a wave every fourth class
constexpr int kDeltaSide = 64, kDeltaFewTiles = 32;
__global__ __launch_bounds__(256) void rows_direct_delta_kernel(DirectArgs a)
{
    __shared__ float2 red[4][kDeltaSide];
    __shared__ float tile[kDeltaSide][kDeltaSide + 1];
    __shared__ double shares[kDeltaSide];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int v0 = blockIdx.y * kDeltaSide;
    constexpr float kNone = -__builtin_inff();
    float db = 0.f;
    double share = 0.0;
    for (int i = 0; i < a.batch; ++i) {
        const int n = (blockIdx.x * a.batch + i) * kDeltaSide + lane, at = n < a.N ? n : a.N - 1;
        if (n - lane >= a.N) break;                      // (uniform)
        float x[16];
        if (a.delta)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int v = v0 + wave + 4 * k;
                x[k] = a.scores[(v < a.V ? v : a.V - 1) * a.score_row + at];
            }
        const float w = row_weight(a.mask, at), weight = n < a.N ? w : 0.f;
        const int label = weight != 0.f ? a.mask.labels[at] : kNoLabel;
        float lse;
        if (a.tiles > kDeltaFewTiles) {                  // joined before
            lse = a.lse[at];
        } else {
            float2 t[kDeltaFewTiles / 4], s{kNone, 0.f};
#pragma unroll
            for (int q = 0; q < kDeltaFewTiles / 4; ++q) {
                const int of = wave + 4 * q;
                t[q] = a.stats[(long)(of < a.tiles ? of : 0) * a.N + at];
            }
#pragma unroll
            for (int q = 0; q < kDeltaFewTiles / 4; ++q)
                if (wave + 4 * q < a.tiles) s = direct_join(s, t[q]);
            red[wave][lane] = s;
            __syncthreads();
            s = red[0][lane];
#pragma unroll
            for (int q = 1; q < 4; ++q) s = direct_join(s, red[q][lane]);
            lse = s.x == kNone ? kNone : s.x + logf(s.y);
            if (blockIdx.y == 0 && wave == 0 && n < a.N) {
                float loss = 0.f;
                if (weight != 0.f) {
                    const float score = a.label_score[n];
                    loss = weight * (score == kNone ? __builtin_inff() : lse - score);   // (a class that is switched off)
                }
                if (a.rowloss) a.rowloss[n] = loss;
                if (a.lse_out) a.lse_out[n] = weight != 0.f ? lse : 0.f;
                if (a.weight) a.weight[n] = weight;
                share += (double)loss;
            }
        }
        if (!a.delta) {                                  // the loss alone
            __syncthreads();                             // (`red` has been read)
            continue;
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const int v = v0 + wave + 4 * k;
            const float g = class_delta(x[k], lse, label != kNoLabel, label == v) * weight, put = weight != 0.f ? g : 0.f;
            tile[wave + 4 * k][lane] = put;
            if (v < a.V) a.scores[v * a.score_row + n] = put;
        }
        __syncthreads();
        if (a.db) {                                      // four threads a class
            float s = 0.f;
#pragma unroll
            for (int z = 0; z < 16; ++z) s += tile[tid >> 2][16 * (tid & 3) + z];
            db += s;
        }
        __syncthreads();
    }
    if (a.db) {
        db += __shfl_xor(db, 1, 64);
        db += __shfl_xor(db, 2, 64);
        const int v = v0 + (tid >> 2);
        if ((tid & 3) == 0 && v < a.V) (a.db_part ? a.db_part + (long)blockIdx.x * a.V : a.db)[v] = db;
    }
    if (blockIdx.y == 0 && a.shares) {
        if (wave == 0) shares[lane] = share;
        __syncthreads();
        if (tid == 0) {
            double s = 0.0;
            for (int q = 0; q < kDeltaSide; ++q) s += shares[q];
            a.shares[blockIdx.x] = s;
        }
    }
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
    if (!dx && id >= a.w_groups) {                       // bias gradients: 32 classes, the parts dealt to eight threads each
        id -= a.w_groups;
        if (id >= a.db_groups) return;                   // (a launch for the loss alone)
        float (*const db_red)[32] = reinterpret_cast<float (*)[32]>(fold);
        const int own = tid & 31, deal = tid >> 5;
        const long v = (long)id * 32 + own;
        float s = 0.f;
        if (v < a.V) {
            int i = deal;
            for (; i + 56 < a.db_parts; i += 64) {
                float u[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) u[q] = a.db_part[(long)(i + 8 * q) * a.V + v];
#pragma unroll
                for (int q = 0; q < 8; ++q) s += u[q];
            }
            for (; i < a.db_parts; i += 8) s += a.db_part[(long)i * a.V + v];
        }
        db_red[deal][own] = s;
        __syncthreads();
        if (deal == 0 && v < a.V) {
            for (int q = 1; q < 8; ++q) s += db_red[q][own];
            a.db[v] = s;
        }
        return;
    }
    const bool deal = (dx ? a.x_deal : a.w_deal) == 4;
    const int splits = dx ? a.x_splits : a.w_splits, each = dx ? a.x_each : a.w_each, along = dx ? a.x_along : a.w_along;
    const int K = dx ? a.V : a.N, M = dx ? a.N : a.V;
    const int tile = id / splits, split = id - tile * splits;
    const int mt = tile / along, dt = tile - mt * along;
    const int side = deal ? 32 : 64;
    const int m0 = mt * side + (deal ? 0 : 32 * (wave >> 1)), d0 = dt * side + (deal ? 0 : 32 * (wave & 1)), k0 = split * each;
    const int len = K - k0 < each ? K - k0 : each, steps = (len + kDirectK - 1) / kDirectK, full = len / kDirectK;
    const int first = deal ? wave : 0, by = deal ? 4 : 1;
    v16f acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    const int d = d0 + row < a.D ? d0 + row : a.D - 1;
    const int m = m0 + row < M ? m0 + row : M - 1;
    // fetches across the rows of memory (weights, features, and the derivative for dx): lanes side by side, 8 k's one below the other
    const T* const b = dx ? (const T*)a.w : (const T*)a.x;
    const long b_pitch = dx ? a.w_pitch : a.x_pitch;
    const T* const bp = b + (k0 + 8 * half) * b_pitch + d;
    auto fetch_b = [&](T (&y)[16], int s) {
        if (s < full) {
            const T* const p = bp + s * kDirectK * b_pitch;
#pragma unroll
            for (int z = 0; z < 16; ++z) y[z] = p[(16 * (z >> 3) + (z & 7)) * b_pitch];
        } else {
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int k = k0 + s * kDirectK + 16 * (z >> 3) + 8 * half + (z & 7);
                y[z] = b[(k < K ? k : K - 1) * b_pitch + d];
            }
        }
    };
    if (dx) {
        const float* const ap = a.scores + (k0 + 8 * half) * a.score_row + m;
        float u[16];
        T y[16];
        auto fetch = [&](int s) {
            if (s < full) {
                const float* const p = ap + s * kDirectK * a.score_row;
#pragma unroll
                for (int z = 0; z < 16; ++z) u[z] = p[(16 * (z >> 3) + (z & 7)) * a.score_row];
            } else {
#pragma unroll
                for (int z = 0; z < 16; ++z) {
                    const int k = k0 + s * kDirectK + 16 * (z >> 3) + 8 * half + (z & 7);
                    u[z] = a.scores[(k < K ? k : K - 1) * a.score_row + m];
                }
            }
            fetch_b(y, s);
        };
        if (first < steps) fetch(first);
        for (int s = first; s < steps; s += by) {
            v8f p[2], q[2];
            const int left = len - s * kDirectK;
#pragma unroll
            for (int z = 0; z < 16; ++z) {
                const int k = 16 * (z >> 3) + 8 * half + (z & 7);
                p[z >> 3][z & 7] = k < left ? u[z] : 0.f;
                q[z >> 3][z & 7] = (float)y[z];          // (beyond the last class times a derivative of zero: finite or not finite anyway)
            }
            if (s + by < steps) fetch(s + by);
            direct_product<kDeltaParts<T>, kParts<T>>(acc, p[0], q[0]);
            direct_product<kDeltaParts<T>, kParts<T>>(acc, p[1], q[1]);
        }
    } else {
        const float* const ap = a.scores + m * a.score_row;
        v8f u[2];
        T y[16];
        auto fetch = [&](int s) {
#pragma unroll
            for (int k = 0; k < 2; ++k) u[k] = load8(ap + k0 + s * kDirectK + 16 * k + 8 * half);   // (padded to whole steps with zeros)
            fetch_b(y, s);
        };
        if (first < steps) fetch(first);
        for (int s = first; s < steps; s += by) {
            v8f p[2], q[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                p[k] = u[k];
#pragma unroll
                for (int z = 0; z < 8; ++z) q[k][z] = (float)y[8 * k + z];
            }
#pragma unroll
            for (int z = 0; z < 16; ++z) {               // rows that add nothing may hold anything
                const int n = k0 + s * kDirectK + 16 * (z >> 3) + 8 * half + (z & 7);
                if (a.weight[n < K ? n : K - 1] == 0.f) q[z >> 3][z & 7] = 0.f;
            }
            if (s + by < steps) fetch(s + by);
            direct_product<kDeltaParts<T>, kParts<T>>(acc, p[0], q[0]);
            direct_product<kDeltaParts<T>, kParts<T>>(acc, p[1], q[1]);
        }
    }

    auto put = [&](int m, int d, float v) {
        if (m >= M || d >= a.D) return;
        if (splits > 1) {
            (dx ? a.x_part : a.w_part)[((long)split * M + m) * a.D + d] = v;
        } else if (dx) {
            store1((T*)a.dx + m * a.dx_pitch + d, a.weight[m] == 0.f ? 0.f : v);
        } else {
            store1((T*)a.dw + (long)m * a.D + d, v);
        }
    };
    if (deal) {
        const v4f s = direct_fold(acc, fold);
#pragma unroll
        for (int q = 0; q < 4; ++q) put(m0 + 4 * (tid >> 5) + q, d0 + (tid & 31), s[q]);
        return;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) put(m0 + 8 * (r >> 2) + 4 * half + (r & 3), d0 + row, acc[r]);
}

template <typename T>
__global__ __launch_bounds__(256) void rows_direct_sum_kernel(DirectArgs a)
{
    const long nx = a.x_part ? (long)a.N * a.D : 0, nw = a.w_part ? (long)a.V * a.D : 0;
    for (long e = (long)blockIdx.x * 256 + threadIdx.x; e < nx + nw; e += (long)gridDim.x * 256) {
        const bool of_x = e < nx;
        const long at = of_x ? e : e - nx, by = of_x ? nx : nw;
        const float* const part = (of_x ? a.x_part : a.w_part) + at;
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
            store1((T*)a.dx + n * a.dx_pitch + (at - n * a.D), a.weight[n] == 0.f ? 0.f : s);
        } else {
            store1((T*)a.dw + at, s);
        }
    }
}

}  // namespace mpcnn
