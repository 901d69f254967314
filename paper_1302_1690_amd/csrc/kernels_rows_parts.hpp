// Around the matrix products of the class layer on rows of features (class_rows.hip): operands brought into blocks of 16-bit numbers, as they
// are and transposed; the softmax's statistics joined; scores turned into the loss's derivative; partial sums added up.
// All of it is bound by memory: 64 x 64 tiles through LDS, each number read once and written in both orders where both are needed.
// 4100 x 16001 scores into the derivative 100 us (5.2 TB/s), 8192 x 4096 bf16 transposed 31 us (4.3), the magnitudes of 4100 x 768 and 16001 x 768 fp32
// 20 us (3.1, from the cache in part), partial sums of 8192 x 4096 x 1 92 us, statistics of 4100 rows 8 us.
#pragma once
#include "any_address.hpp"
#include "ranges.hpp"
#include "rows_mask.hpp"

namespace mpcnn {

constexpr int kPeakGroups = 256;           // words of a peak
constexpr int kDeltaRaise = 14;            // what the derivative (up to 1) is raised by

// ---- the largest magnitude of a matrix, as bits (one word per workgroup); what is not finite is passed over
struct PeakArgs {
    const float* src;
    long pitch;
    long rows;
    int cols;
    RowMask mask;                          // labels null: every row
    int weighted;                          // numbers times their row's weight
    unsigned* words;                       // [kPeakGroups]
};
struct PeakSet { PeakArgs of[3]; };        // blockIdx.y: which
__global__ __launch_bounds__(1024) void rows_peak_kernel(PeakSet set)
{
    __shared__ unsigned red[16];
    const PeakArgs& a = set.of[blockIdx.y];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned peak = 0;
    auto add = [&](const v8f& x, float weight) {
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            const unsigned b = bits_of(x[z] * (a.weighted ? weight : 1.f)) & 0x7fffffffu;
            peak = weight != 0.f && b < kNoPeak && b > peak ? b : peak;
        }
    };
    // eight numbers of a row at a time, four times eight in flight; rows without gaps are one (whose last eight numbers' end is a 32-bit number, too)
    const bool one = a.pitch == a.cols && !a.mask.labels && a.rows * a.cols <= 0x7fffffff - 8;
    const long cols = one ? a.rows * a.cols : a.cols, rows = one ? 1 : a.rows;
    const long octets = (cols + 7) / 8, all = rows * octets, step = (long)gridDim.x * 1024;
    for (long e = (long)blockIdx.x * 1024 + threadIdx.x; e < all; e += 4 * step) {
        v8f v[4];
        float weight[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const long at = e + q * step < all ? e + q * step : e;
            const long r = all == octets ? 0 : at / octets, c = 8 * (at - r * octets);
            v[q] = load8_of(a.src + r * a.pitch, (int)c, (int)cols);
            weight[q] = a.mask.labels ? row_weight(a.mask, (int)r) : 1.f;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) add(v[q], weight[q]);
    }
    peak = wave_largest(peak);
    if (lane == 0) red[wave] = peak;
    __syncthreads();
    if (threadIdx.x == 0) {
        unsigned m = red[0];
        for (int w = 1; w < 16; ++w) m = red[w] > m ? red[w] : m;
        a.words[blockIdx.x] = m;
    }
}

// ---- blocks: 64 bf16 numbers, or the two parts of 32 fp32 ones (kernels_rows_product.hpp)
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Piece p (16 bytes) of the 128 (bf16) or 256 (parts) bytes that 64 numbers take; get(i) is the i-th of them, raised; second parts by low_up more
template <bool HALVES, typename F>
__device__ __forceinline__ v4f piece_of(int p, F get, float low_up = 1.f)
{
    if constexpr (HALVES) {
        f16x8_t v;
        const int at = 32 * (p >> 3) + 8 * (p & 3);
        const bool low = (p & 4) != 0;
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            const float x = get(at + z);
            const _Float16 h = (_Float16)x;
            v[z] = low ? (_Float16)((x - (float)h) * low_up) : h;
        }
        return __builtin_bit_cast(v4f, v);
    } else {
        bf16x8_t v;
#pragma unroll
        for (int z = 0; z < 8; ++z) v[z] = (__bf16)get(8 * p + z);
        return __builtin_bit_cast(v4f, v);
    }
}

// ---- a matrix [R][C] into blocks along its rows (`rows`: [R][row_bytes]) and along its columns (`cols`: [C][col_bytes]), either may be null.
// Padding is zero, rows that add nothing are too.
struct PackRowsArgs {
    const void* src;
    long pitch;                            // elements
    int R, C;
    char *rows, *cols;
    long row_bytes, col_bytes;
    RowMask mask;                          // labels null: every row
    const unsigned *peak, *col_peak;       // fp32: [kPeakGroups], what the numbers are raised by; along the columns they are times their row's weight
};
// fp32, two parts
__global__ __launch_bounds__(256) void rows_pack_kernel(PackRowsArgs a)
{
    constexpr int kPieces = 16;
    __shared__ float tile[64][65];
    const int c0 = 64 * blockIdx.y, r0 = 64 * blockIdx.x;
    __shared__ float weight[64];
    const float up = power_of_two(raise_of(peak_of(a.peak, kPeakGroups), 0));
    v8f v[2];
    float w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {                        // 8 lanes a row, 8 numbers each
        const int r = r0 + 32 * i + (threadIdx.x >> 3), at = r < a.R ? r : a.R - 1;
        v[i] = load8_of((const float*)a.src + at * a.pitch, c0 + 8 * (threadIdx.x & 7), a.C);
        const float of = a.mask.labels ? row_weight(a.mask, at) : 1.f;
        w[i] = r < a.R ? of : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 32 * i + (threadIdx.x >> 3);
#pragma unroll
        for (int z = 0; z < 8; ++z) tile[r][8 * (threadIdx.x & 7) + z] = w[i] != 0.f ? v[i][z] : 0.f;
        if ((threadIdx.x & 7) == 0) weight[r] = w[i];
    }
    __syncthreads();
    if (a.rows)
        for (int q = threadIdx.x; q < 64 * kPieces; q += 256) {
            const int r = q / kPieces, p = q % kPieces;
            const long at = (long)blockIdx.y * (kPieces * 16) + 16 * p;
            if (r0 + r >= a.R || at >= a.row_bytes) continue;
            *reinterpret_cast<v4f*>(a.rows + (long)(r0 + r) * a.row_bytes + at) = piece_of<true>(p, [&](int i) { return tile[r][i] * up; });
        }
    if (a.cols) {
        const float up_c = power_of_two(raise_of(peak_of(a.col_peak, kPeakGroups), 0));
        for (int q = threadIdx.x; q < 64 * kPieces; q += 256) {
            const int c = q / kPieces, p = q % kPieces;
            const long at = (long)blockIdx.x * (kPieces * 16) + 16 * p;
            if (c0 + c >= a.C || at >= a.col_bytes) continue;
            *reinterpret_cast<v4f*>(a.cols + (long)(c0 + c) * a.col_bytes + at) = piece_of<true>(p, [&](int i) { return tile[i][c] * weight[i] * up_c; });
        }
    }
}
// bf16: as they are, 128 rows per workgroup.  LDS holds pairs of columns; a thread reads 8 rows of a pair and leaves a piece of either column.
__global__ __launch_bounds__(256) void rows_pack16_kernel(PackRowsArgs a)
{
    typedef unsigned v4u __attribute__((ext_vector_type(4)));
    __shared__ unsigned tile[128][33];
    const int c0 = 64 * blockIdx.y, r0 = 128 * blockIdx.x;
    v4u v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                        // 8 lanes a row, 8 numbers each
        const int r = r0 + 32 * i + (threadIdx.x >> 3), at = r < a.R ? r : a.R - 1;
        const Raw8<bf16> u = raw8_of((const bf16*)a.src + at * a.pitch, c0 + 8 * (threadIdx.x & 7), a.C);
        const bool there = r < a.R && (!a.mask.labels || row_weight(a.mask, at) != 0.f);
        v[i] = there ? __builtin_bit_cast(v4u, u.a) : v4u{0, 0, 0, 0};
    }
    if (a.rows)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 32 * i + (threadIdx.x >> 3);
            const long at = (long)blockIdx.y * 128 + 16 * (threadIdx.x & 7);
            if (r < a.R && at < a.row_bytes) *reinterpret_cast<v4u*>(a.rows + (long)r * a.row_bytes + at) = v[i];
        }
    if (!a.cols) return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int z = 0; z < 4; ++z) tile[32 * i + (threadIdx.x >> 3)][4 * (threadIdx.x & 7) + z] = v[i][z];
    __syncthreads();
    const int oct = threadIdx.x & 15;
    const long at = (long)blockIdx.x * 256 + 16 * oct;
    if (at >= a.col_bytes) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int pair = 16 * i + (threadIdx.x >> 4), c = c0 + 2 * pair;
        unsigned x[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) x[z] = tile[8 * oct + z][pair];
        v4u even, odd;
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            even[z] = (x[2 * z] & 0xffffu) | x[2 * z + 1] << 16;
            odd[z] = x[2 * z] >> 16 | (x[2 * z + 1] & 0xffff0000u);
        }
        if (c < a.C) *reinterpret_cast<v4u*>(a.cols + (long)c * a.col_bytes + at) = even;
        if (c + 1 < a.C) *reinterpret_cast<v4u*>(a.cols + (long)(c + 1) * a.col_bytes + at) = odd;
    }
}

// ---- scores from the partial sums of their product: their statistics over 32 classes, their label's, and the scores themselves where they are kept
struct ScoresSumArgs {
    const float* part;                     // [splits][M][N]
    int splits, M, N;
    const unsigned *a_peak, *b_peak;       // fp32 storage: what the operands were raised by
    const float* bias;                     // [M] or null
    const int* labels;                     // [N]
    float2* stats;                         // [tiles of 32 classes][N]
    float* label_score;                    // [N]
    float* scores;                         // [M][score_row], or null
    long score_row;
};
constexpr int kScoresSum = 32;            // classes of a workgroup, eight a wave
template <bool HALVES>
__global__ __launch_bounds__(256) void rows_scores_sum_kernel(ScoresSumArgs a)
{
    constexpr float kNone = -__builtin_inff();
    __shared__ float2 red[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = 64 * blockIdx.x + lane, at = n < a.N ? n : a.N - 1, m0 = kScoresSum * blockIdx.y + wave;
    Lower f{1.f, 1.f};
    if constexpr (HALVES) f = lower_by(raise_of(peak_of(a.a_peak, kPeakGroups), 0) + raise_of(peak_of(a.b_peak, kPeakGroups), 0));
    float s[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] = 0.f;
    const float* p[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = a.part + (long)(m0 + 4 * k < a.M ? m0 + 4 * k : a.M - 1) * a.N + at;
    const long by = (long)a.M * a.N;
    int i = 0;
    for (; i + 4 <= a.splits; i += 4) {                  // 32 loads in flight
        float v[4][8];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[q][k] = p[k][(i + q) * by];
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] += v[q][k];
    }
    for (; i < a.splits; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += p[k][i * by];
    const int label = n < a.N ? a.labels[n] : -1;
    float top = kNone;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int m = m0 + 4 * k;
        if constexpr (HALVES) s[k] = s[k] * f.first * f.second;
        s[k] = m < a.M ? s[k] + (a.bias ? a.bias[m] : 0.f) : kNone;
        top = fmaxf(top, s[k]);
        if (m >= a.M || n >= a.N) continue;
        if (a.scores) a.scores[m * a.score_row + n] = s[k];
        if (m == label) a.label_score[n] = s[k];
    }
    const float base = top == kNone ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += __expf(s[k] - base);
    red[wave][lane] = float2{top, sum};
    __syncthreads();
    if (wave != 0 || n >= a.N) return;
    float2 t = red[0][lane];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        const float2 o = red[w][lane];
        const float all = fmaxf(t.x, o.x), b = all == kNone ? 0.f : all;
        t = float2{all, t.y * __expf(t.x - b) + o.y * __expf(o.x - b)};
    }
    a.stats[(long)blockIdx.y * a.N + n] = t;
}

// ---- per row: the statistics of all tiles of classes joined; the loss; per workgroup its share of the summed loss
struct JoinArgs {
    const float2* stats;                   // [tiles][N]
    int tiles, N;
    const float* label_score;              // [N]
    RowMask mask;
    float *lse, *rowloss, *weight;         // [N]: lse for the derivative, results (null: not asked for), the row's weight or 0
    float* lse_out;
    double* loss_part;                     // per workgroup, or null
};
// ROWS rows per workgroup, the tiles dealt to THREADS / ROWS threads each.  Up to 8 rows, or 32 with few tiles: one workgroup, whose loss is the
// whole one; 4 rows while that leaves compute units without work; 32 beyond (whole lines).
constexpr int kJoinLeast = 8, kJoinFew = 4, kJoinMany = 32, kJoinFewMost = 1024, kJoinTiles = 512;
inline int join_rows(int N, int tiles)
{
    return N <= kJoinLeast ? kJoinLeast : N <= kJoinMany && tiles <= kJoinTiles ? kJoinMany : N <= kJoinFewMost ? kJoinFew : kJoinMany;
}
template <int ROWS, int THREADS>
__global__ __launch_bounds__(THREADS) void rows_join_kernel(JoinArgs a)
{
    constexpr int DEALS = THREADS / ROWS;
    __shared__ float2 red[DEALS][ROWS];
    __shared__ double sums[ROWS];
    const int own = threadIdx.x % ROWS, deal = threadIdx.x / ROWS;
    const int n = blockIdx.x * ROWS + own;
    constexpr float kNone = -__builtin_inff();
    auto join = [](float2 s, float2 o) {
        const float top = fmaxf(s.x, o.x), base = top == kNone ? 0.f : top;
        return float2{top, s.y * __expf(s.x - base) + o.y * __expf(o.x - base)};
    };
    float2 s{kNone, 0.f};
    if (n < a.N) {
        // (fp64: of hundreds of millions of classes there are a hundred thousand tiles a thread, each below half a step of an fp32 sum that has one likely class)
        double sum = 0.0;
        auto add = [&](float2 o) {
            const float top = fmaxf(s.x, o.x), base = top == kNone ? 0.f : top;
            sum = fma(sum, (double)__expf(s.x - base), (double)(o.y * __expf(o.x - base)));
            s.x = top;
        };
        int t = deal;
        for (; t + 7 * DEALS < a.tiles; t += 8 * DEALS) {
            float2 v[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = a.stats[(long)(t + DEALS * q) * a.N + n];
#pragma unroll
            for (int q = 0; q < 8; ++q) add(v[q]);
        }
        for (; t < a.tiles; t += DEALS) add(a.stats[(long)t * a.N + n]);
        s.y = (float)sum;
    }
    red[deal][own] = s;
    __syncthreads();
    for (int w = DEALS / 2; w >= 8; w >>= 1) {   // (a tree down to eight, in a fixed order)
        if (deal < w) red[deal][own] = join(red[deal][own], red[deal + w][own]);
        __syncthreads();
    }
    s = red[0][own];
    if (deal == 0) {
        double share = 0.0;
        if (n < a.N) {
            for (int d = 1; d < 8; ++d) s = join(s, red[d][own]);
            const float lse = s.x == kNone ? kNone : s.x + logf(s.y);
            const float w = row_weight(a.mask, n);
            float loss = 0.f;
            if (w != 0.f) {
                const float score = a.label_score[n];
                loss = w * (score == kNone ? __builtin_inff() : lse - score);   // (a class that is switched off)
            }
            if (a.lse) a.lse[n] = lse;
            if (a.weight) a.weight[n] = w;
            if (a.lse_out) a.lse_out[n] = w != 0.f ? lse : 0.f;
            if (a.rowloss) a.rowloss[n] = loss;
            share = (double)loss;
        }
        sums[own] = share;
    }
    if (!a.loss_part) return;
    __syncthreads();
    if (threadIdx.x == 0) {
        double all = 0.0;
        for (int i = 0; i < ROWS; ++i) all += sums[i];
        a.loss_part[blockIdx.x] = all;
    }
}

// ---- scores [classes][score_row] of a piece of the classes into the derivative p - [class = label], in blocks along the rows ([classes][out_bytes]):
// with bf16 storage times the row's weight (rounded once), with fp32 storage raised by 2^kDeltaRaise, its second parts by kLowUp more (kernels_rows_product.hpp; the
// weight follows: with the features, or behind the product).  db_part: per tile of 64 rows the sums over them, weighted.
struct DeltaArgs {
    const float* scores;
    long score_row;
    int classes, class0, N;
    const int* labels;
    const float *lse, *weight;             // [N]
    char* out;                             // or null
    long out_bytes;
    float* db_part;                        // [tiles of rows][classes], or null
};
template <bool HALVES>
__global__ __launch_bounds__(256) void rows_delta_kernel(DeltaArgs a)
{
    constexpr int kPieces = HALVES ? 16 : 8;
    __shared__ float tile[64][65];
    __shared__ float weight[64];
    __shared__ float sums[4][64];
    const int n0 = 64 * blockIdx.x, v0 = 64 * blockIdx.y;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = n0 + lane;
    const bool real = n < a.N;
    const float w = real ? a.weight[n] : 0.f, lse = real ? a.lse[n] : 0.f;
    const int label = real ? a.labels[n] - a.class0 : -1;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int v = v0 + wave + 4 * i;
        x[i] = v < a.classes && w != 0.f ? a.scores[(long)v * a.score_row + n] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int v = v0 + wave + 4 * i;
        float g = 0.f;
        if (v < a.classes && w != 0.f) {
            g = class_delta(x[i], lse, true, v == label);
            if constexpr (!HALVES) g *= w;
        }
        tile[wave + 4 * i][lane] = g;
    }
    if (wave == 0) weight[lane] = HALVES ? w : 1.f;
    __syncthreads();
    if (a.db_part) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += tile[lane][16 * wave + i] * weight[16 * wave + i];
        sums[wave][lane] = s;
    }
    if (a.out)
        for (int q = threadIdx.x; q < 64 * kPieces; q += 256) {
            const int c = q / kPieces, p = q % kPieces;
            const long at = (long)blockIdx.x * (kPieces * 16) + 16 * p;
            if (v0 + c >= a.classes || at >= a.out_bytes) continue;
            *reinterpret_cast<v4f*>(a.out + (long)(v0 + c) * a.out_bytes + at) = piece_of<HALVES>(p, [&](int i) { return HALVES ? tile[c][i] * power_of_two(kDeltaRaise) : tile[c][i]; }, kLowUp);
        }
    if (a.db_part) {
        __syncthreads();
        if (wave == 0 && v0 + lane < a.classes)
            a.db_part[(long)blockIdx.x * a.classes + v0 + lane] = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    }
}

// ---- partial sums [splits][M][N] of a product added up, lowered, scaled and rounded
struct SumArgs {
    const float* part;
    int splits;
    long M, N, out_row;
    const unsigned* b_peak;                // as in ProductArgs, of the derivative's products
    int halves;
    const float* row_scale;
    int row_mask;
    void* out;
    int out_bf16;
};
__global__ __launch_bounds__(256) void rows_sum_kernel(SumArgs a)
{
    Lower f{1.f, 1.f};
    if (a.halves) f = lower_by(kDeltaRaise + raise_of(peak_of(a.b_peak, kPeakGroups), 0));
    const long all = a.M * a.N;
    for (long e = (long)blockIdx.x * 256 + threadIdx.x; e < all; e += (long)gridDim.x * 256) {
        double s = 0.0;
        for (int i = 0; i < a.splits; ++i) s += (double)a.part[i * all + e];
        const long m = e / a.N, n = e - m * a.N;
        float scale = a.row_scale ? a.row_scale[m] : 1.f;
        scale = a.row_mask && scale != 0.f ? 1.f : scale;
        const float v = scale == 0.f ? 0.f : (float)s * f.first * f.second * scale;
        if (a.out_bf16) ((bf16*)a.out)[m * a.out_row + n] = (bf16)v;
        else ((float*)a.out)[m * a.out_row + n] = v;
    }
}

// ---- no rows: gradients and loss are zero
__global__ __launch_bounds__(256) void rows_none_kernel(char* dw, long bytes, float* db, long classes, double* loss)
{
    const long at = (long)blockIdx.x * 256 + threadIdx.x, step = (long)gridDim.x * 256;
    if (dw)
        for (long e = at; e < bytes / 2; e += step) reinterpret_cast<unsigned short*>(dw)[e] = 0;
    if (db)
        for (long e = at; e < classes; e += step) db[e] = 0.f;
    if (loss && at == 0) *loss = 0.0;
}

// ---- bias gradients from the sums per tile of rows; the summed loss (workgroup 0); both in a fixed order
struct FinishArgs {
    const float* db_part;                  // [tiles][classes]
    int tiles;
    long classes;
    float* db;                             // or null
    const double* loss_part;
    int loss_parts;
    double* loss;                          // or null
};
__global__ __launch_bounds__(256) void rows_finish_kernel(FinishArgs a)
{
    __shared__ double red[256];
    if (blockIdx.x == 0 && a.loss) {
        double s = 0.0;
        for (int i = threadIdx.x; i < a.loss_parts; i += 256) s += a.loss_part[i];
        red[threadIdx.x] = s;
        __syncthreads();
        for (int w = 128; w > 0; w >>= 1) {
            if ((int)threadIdx.x < w) red[threadIdx.x] += red[threadIdx.x + w];
            __syncthreads();
        }
        if (threadIdx.x == 0) *a.loss = red[0];
    }
    if (!a.db) return;
    __syncthreads();
    // 32 classes, the tiles dealt to eight threads each, eight loads in flight
    const int own = threadIdx.x & 31, deal = threadIdx.x >> 5;
    const long v = (long)blockIdx.x * 32 + own;
    double s = 0.0;
    if (v < a.classes) {
        int t = deal;
        for (; t + 56 < a.tiles; t += 64) {
            float u[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) u[q] = a.db_part[(long)(t + 8 * q) * a.classes + v];
#pragma unroll
            for (int q = 0; q < 8; ++q) s += (double)u[q];
        }
        for (; t < a.tiles; t += 8) s += (double)a.db_part[(long)t * a.classes + v];
    }
    red[threadIdx.x] = s;
    __syncthreads();
    if (deal != 0 || v >= a.classes) return;
    for (int q = 1; q < 8; ++q) s += red[32 * q + own];
    a.db[v] = (float)s;
}

}  // namespace mpcnn
