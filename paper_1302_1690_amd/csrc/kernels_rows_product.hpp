// The matrix product of the class layer on rows of features (class_rows.hip): C[m][n] = sum_k A[m][k] B[n][k], 16-bit numbers on
// v_mfma_f32_32x32x16, sums in fp32; both operands with k running fastest, or (ACROSS) both with k as the rows of memory, A[k][m], B[k][n].
//
// Operands.  bf16 storage: as they are.  fp32 storage: two fp16 parts per number (x 2^e = h + l, ranges.hpp), which lie in turn,
// 32 numbers' first parts and their second parts, so that one 128-byte block of a row is 64 bf16 numbers or 32 fp32 ones and the kernel's
// fetches are the same; the products are h h', h l' and l h' (what is left out, l l', is below 2^-22 of a product).  The derivative is p for all but
// the labels' classes, and with many classes most p are far below the scale that suits the labels' (numbers up to 1 are raised by 2^14): its second parts
// are raised by 2^11 more (kLowUp), and what they are multiplied with, the first parts of the class weights or the features, is lowered by as much in
// registers.  Then it keeps 22 bits down to 2^-28, and is off by at most 2^-49 below (without: 2^-17, 2^-39; a class that is nobody's label and has p = 1e-9 got a
// gradient that was off by 1e-3).  With bf16 storage the derivative times the row's weight is one bf16 number: the
// gradients' error against 64 bits, 1.65e-3 of them by their own rounding (2-norm), grows to 1.68e-3 (8192 x 4096 x 128000) .. 1.89e-3 (816 x 1059 x 3465), with row weights to 2.3e-3; a
// second part would make both gradients' products twice as long.  k is padded with zeros to whole blocks; rows beyond the last are not read (the last one is, again, and its results dropped).
//
// A workgroup computes a tile of 32 WM MT x 32 WN NT results, each wave MT x NT of the instruction's, in accumulators.  Both operands' next
// blocks come from memory straight into the LDS buffer that is not being multiplied (128 bits per lane, a barrier per block).  An LDS row is a
// block (128 bytes); its 16-byte pieces lie permuted by half the row's number (two rows are the 256 bytes of the banks), so that the lanes of an
// operand's fetch, which read one piece each of 32 rows, find them on different banks.  The permutation is made by the addresses in memory that the lanes fetch from.
//
// ACROSS: a block is 64 k's (32 of fp32 storage) of the tile's columns, an LDS row a k's 512 bytes (for 128 columns 256, of fp32 storage twice
// that).  The instruction wants 8 k's of one column per lane: ds_read_b64_tr_b16 turns 4 k's x 16 columns around within 16 lanes (lane r names
// 4 columns, r % 4, of k r / 4 and receives column r at all 4), so two of them are an operand.  The 4 k's 64 bytes, which 32 lanes fetch
// together, lie permuted by k (64-byte groups), on different banks.  Rows of k beyond the last come as zeros (the descriptor's bound).
//
// Results: the classes' scores with their bias (m = class, n = row), of which only each row's largest and sum of exponentials over the
// tile's classes leave the kernel (and the score of its label), or which are stored too; or the loss's derivative in the place of the scores, as
// the gradients' products want it; or products, stored rounded; or partial sums.
//
// Bound by the matrix instruction at the clock that its power leaves (a library's plain bf16 product reaches 1.21-1.29 PFLOP/s, this layer's fp32
// products a third of that).  8192 x 4096 x 32000 bf16, 2.1e12 operations: scores' statistics 1.78 ms (1.21 PFLOP/s), derivative 1.92 ms (1.12), features'
// gradient 1.82 ms (1.18), class weights' gradient 1.72 ms (1.25).  4100 x 768 x 16001 fp32, 1.0e11: scores, stored, 384 us (262 TFLOP/s), gradients
// 349 (289) and 332 (303).  256 x 256 results on eight waves: half the fetches of 128 x 128, which has more workgroups where there is less work.
#pragma once
#include <type_traits>

#include "any_address.hpp"
#include "kernels_rows_parts.hpp"

namespace mpcnn {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlockBytes = 128;           // of a row of an operand
constexpr float kLog2e = 1.4426950408889634f;

struct ProductArgs {
    const char *A, *B;                     // rows of blocks
    long a_row, b_row;                     // bytes
    long a_bytes, b_bytes;                 // ACROSS: of the operands in all
    int M, N;
    int blocks, per_split;                 // along k: in all, of a workgroup
    int tiles_m, tiles_n, splits;
    const unsigned *a_peak, *b_peak;       // fp32 storage: [kPeakGroups], what the operands were raised by (a_peak null: A is the derivative, kDeltaRaise)
    // scores
    const float* bias;                     // [M] or null
    const int* labels;                     // [N]
    float2* stats;                         // [tiles_m][N]: largest, sum of exp(score - largest)
    float* label_score;                    // [N]
    float* scores;                         // [M][score_row], or null
    long score_row;
    int class0;                            // the first class of A
    // derivative
    const float *lse, *weight;             // [N]
    char* delta;                           // [M][delta_bytes] blocks along the rows, or null
    long delta_bytes;
    int padded;                            // rows, with those of the last block of 64
    float* db_part;                        // [padded / 64][M]: sums over 64 rows, or null
    // products
    void* out;                             // [M][out_row]
    long out_row;
    const float* row_scale;                // [M], or null (0: nothing of the row, whatever it is multiplied with)
    int row_mask;                          // only that
    float* part;                           // [splits][M][N]: partial sums instead (added to what is there: add)
    int add;
};
enum { kScores = 0, kStoreF32 = 1, kStoreBf16 = 2, kPart = 3, kDelta = 4 };

// ACROSS: operands x and y of one step of the instruction, A's from the LDS addresses pa + KA and KA + JA on, B's likewise.  (The builtin for this
// instruction waits for all fetches into LDS, also those into the other buffer: 1144 us against 958 for a product of 8192 x 4096 x 16000.)
template <int KA, int JA, int KB, int JB>
__device__ __forceinline__ void read_turned(v4f (&x)[4], v4f (&y)[2], const unsigned (&pa)[4], const unsigned (&pb)[2])
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    v2f a0, a1, b0, b1, c0, c1, d0, d1, e0, e1, f0, f1;
    asm volatile("ds_read_b64_tr_b16 %0, %12 offset:%18\n\tds_read_b64_tr_b16 %1, %12 offset:%19\n\t"
                 "ds_read_b64_tr_b16 %2, %13 offset:%18\n\tds_read_b64_tr_b16 %3, %13 offset:%19\n\t"
                 "ds_read_b64_tr_b16 %4, %14 offset:%18\n\tds_read_b64_tr_b16 %5, %14 offset:%19\n\t"
                 "ds_read_b64_tr_b16 %6, %15 offset:%18\n\tds_read_b64_tr_b16 %7, %15 offset:%19\n\t"
                 "ds_read_b64_tr_b16 %8, %16 offset:%20\n\tds_read_b64_tr_b16 %9, %16 offset:%21\n\t"
                 "ds_read_b64_tr_b16 %10, %17 offset:%20\n\tds_read_b64_tr_b16 %11, %17 offset:%21\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1), "=&v"(c0), "=&v"(c1), "=&v"(d0), "=&v"(d1), "=&v"(e0), "=&v"(e1), "=&v"(f0), "=&v"(f1)
                 : "v"(pa[0]), "v"(pa[1]), "v"(pa[2]), "v"(pa[3]), "v"(pb[0]), "v"(pb[1]), "n"(KA), "n"(KA + JA), "n"(KB), "n"(KB + JB)
                 : "memory");
    x[0] = v4f{a0[0], a0[1], a1[0], a1[1]}; x[1] = v4f{b0[0], b0[1], b1[0], b1[1]};
    x[2] = v4f{c0[0], c0[1], c1[0], c1[1]}; x[3] = v4f{d0[0], d0[1], d1[0], d1[1]};
    y[0] = v4f{e0[0], e0[1], e1[0], e1[1]}; y[1] = v4f{f0[0], f0[1], f1[0], f1[1]};
}
template <int KA, int JA, int KB, int JB>
__device__ __forceinline__ void read_turned(v4f (&x)[2], v4f (&y)[2], const unsigned (&pa)[2], const unsigned (&pb)[2])
{
    typedef float v2f __attribute__((ext_vector_type(2)));
    v2f a0, a1, b0, b1, e0, e1, f0, f1;
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%14\n\tds_read_b64_tr_b16 %5, %10 offset:%15\n\t"
                 "ds_read_b64_tr_b16 %6, %11 offset:%14\n\tds_read_b64_tr_b16 %7, %11 offset:%15\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1), "=&v"(e0), "=&v"(e1), "=&v"(f0), "=&v"(f1)
                 : "v"(pa[0]), "v"(pa[1]), "v"(pb[0]), "v"(pb[1]), "n"(KA), "n"(KA + JA), "n"(KB), "n"(KB + JB)
                 : "memory");
    x[0] = v4f{a0[0], a0[1], a1[0], a1[1]}; x[1] = v4f{b0[0], b0[1], b1[0], b1[1]};
    y[0] = v4f{e0[0], e0[1], e1[0], e1[1]}; y[1] = v4f{f0[0], f0[1], f1[0], f1[1]};
}

template <int WM, int WN, int MT, int NT, bool HALVES, int RESULT, bool ACROSS>
__global__ __launch_bounds__(64 * WM * WN, 1) void rows_product_kernel(ProductArgs a)
{
    constexpr int BM = 32 * WM * MT, BN = 32 * WN * NT, kWaves = WM * WN;
    constexpr int kStage = (BM + BN) * kBlockBytes;
    constexpr int AI = BM / 8 / kWaves, BI = BN / 8 / kWaves;   // a wave's fetches of 8 rows' blocks
    static_assert(AI * 8 * kWaves == BM && BI * 8 * kWaves == BN && AI % 2 == 0 && BI % 2 == 0, "the waves share the rows evenly");
    extern __shared__ __attribute__((aligned(256))) char lds_raw[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // ---- the workgroup's tile: the XCDs (workgroups go to them in turn) take stretches of the tiles, in groups of 8 tiles along m
    const int tiles = a.tiles_m * a.tiles_n, all = tiles * a.splits;
    const int each = (all + 7) / 8;
    const int t = ((int)blockIdx.x % 8) * each + (int)blockIdx.x / 8;
    if ((int)blockIdx.x / 8 >= each || t >= all) return;
    const int split = t / tiles, tt = t - split * tiles;
    const int group = tt / (8 * a.tiles_n), in = tt - group * 8 * a.tiles_n;
    const int deep = a.tiles_m - 8 * group < 8 ? a.tiles_m - 8 * group : 8;
    const int tn = in / deep, tm = 8 * group + in - tn * deep;
    const int m0 = tm * BM, n0 = tn * BN;

    // ---- fetches: rows 8 q .. 8 q + 7 of a block, lane l the piece l % 8 of row 8 q + l / 8 as it lies in LDS; ACROSS: as many bytes of its rows of k
    typedef __attribute__((address_space(3))) void* lds_ptr;
    constexpr int kSize = HALVES ? 4 : 2, kRows = 64 * 2 / kSize, kARow = BM * kSize, kBRow = BN * kSize;   // ACROSS: bytes of a number, k's of a block, an LDS row
    const int first = split * a.per_split;
    const int count = a.blocks - first < a.per_split ? a.blocks - first : a.per_split;
    const __amdgpu_buffer_rsrc_t ra =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(a.A + (long)m0 * a.a_row + (long)first * kBlockBytes), 0, 0x7fffffff, 0x00020000);
    const __amdgpu_buffer_rsrc_t rb =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(a.B + (long)n0 * a.b_row + (long)first * kBlockBytes), 0, 0x7fffffff, 0x00020000);
    const unsigned piece[2] = {16u * ((lane & 7) ^ (lane >> 4)), 16u * ((lane & 7) ^ (lane >> 4) ^ 4)};   // even, odd q
    unsigned va[AI], vb[BI];
#pragma unroll
    for (int i = 0; i < AI; ++i) {
        if constexpr (ACROSS) {
            const unsigned at = (unsigned)((wave * AI + i) * 1024 + 16 * lane), k = at / kARow;
            va[i] = k * (unsigned)a.a_row + 16u * ((at % kARow / 16) ^ 4 * (k & 3));
        } else {
            const int r = 8 * (wave * AI + i) + (lane >> 3), left = a.M - 1 - m0;
            va[i] = (unsigned)(r < left ? r : left) * (unsigned)a.a_row + piece[i & 1];
        }
    }
#pragma unroll
    for (int i = 0; i < BI; ++i) {
        if constexpr (ACROSS) {
            const unsigned at = (unsigned)((wave * BI + i) * 1024 + 16 * lane), k = at / kBRow;
            vb[i] = k * (unsigned)a.b_row + 16u * ((at % kBRow / 16) ^ 4 * (k & 3));
        } else {
            const int r = 8 * (wave * BI + i) + (lane >> 3), left = a.N - 1 - n0;
            vb[i] = (unsigned)(r < left ? r : left) * (unsigned)a.b_row + piece[i & 1];
        }
    }
    // ACROSS: an operand from a block's first k on (the bound does not see a scalar offset, so each block has a descriptor of its own)
    auto from = [&](const char* operand, long bytes, long offset) {
        const long left = bytes - offset;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(operand + (left > 0 ? offset : 0)), 0,
                                                 left <= 0 ? 0 : left < 0x7fffffff ? (int)left : 0x7fffffff, 0x00020000);
    };
    auto fetch = [&](int block, char* stage) {
        if constexpr (ACROSS) {
            const __amdgpu_buffer_rsrc_t pa = from(a.A, a.a_bytes, (long)(first + block) * kRows * a.a_row + (long)m0 * kSize);
            const __amdgpu_buffer_rsrc_t pb = from(a.B, a.b_bytes, (long)(first + block) * kRows * a.b_row + (long)n0 * kSize);
#pragma unroll
            for (int i = 0; i < AI; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(pa, (lds_ptr)(stage + (wave * AI + i) * 1024), 16, (int)va[i], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < BI; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(pb, (lds_ptr)(stage + BM * kBlockBytes + (wave * BI + i) * 1024), 16, (int)vb[i], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < AI; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(stage + (wave * AI + i) * 1024), 16, (int)va[i], block * kBlockBytes, 0, 0);
#pragma unroll
            for (int i = 0; i < BI; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(stage + BM * kBlockBytes + (wave * BI + i) * 1024), 16, (int)vb[i],
                                                         block * kBlockBytes, 0, 0);
        }
    };

    v16f acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

    // an operand's 16 k's, piece pair s of the block: lane l feeds row l % 32, k's 8 (l / 32) ..
    const int row = lane & 31, half = lane >> 5;
    const int at_a = (32 * MT * wm + row) * kBlockBytes, at_b = (BM + 32 * NT * wn + row) * kBlockBytes, mix = row >> 1 & 7;
    // ACROSS: lane l names 4 columns of k 8 (l / 32) + (l % 16) / 4 of the step's 16, and of the k 4 on
    const int turn = (lane & 15) >> 2, of_row = 8 * half + turn, of_col = 32 * (lane >> 4 & 1) + 8 * (lane & 3);
    int group_a[MT], group_b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) group_a[i] = of_row * kARow + of_col + 64 * ((MT * wm + i) * (HALVES ? 2 : 1) ^ turn);
#pragma unroll
    for (int j = 0; j < NT; ++j) group_b[j] = BM * kBlockBytes + of_row * kBRow + of_col + 64 * ((NT * wn + j) * (HALVES ? 2 : 1) ^ turn);
    // fp32 gradients: by what the partners of A's second parts are lowered, where A is the derivative (else A has a peak of its own)
    constexpr bool kGradient = HALVES && (RESULT == kStoreF32 || RESULT == kPart);
    const _Float16 low = (_Float16)(kGradient && (RESULT == kStoreF32 || ACROSS || !a.a_peak) ? kLowDown : 1.f);
    auto lower = [&](v4f (&y)[NT]) {
#pragma unroll
        for (int j = 0; j < NT; ++j) y[j] = __builtin_bit_cast(v4f, __builtin_bit_cast(f16x8, y[j]) * low);
    };
    auto multiply = [&](const char* stage) {
        auto read = [&](int at, int s) { return *reinterpret_cast<const v4f*>(stage + at + 16 * ((2 * s + half) ^ mix)); };
        auto read_a = [&](int i, int s) { return read(at_a + i * 32 * kBlockBytes, s); };
        auto read_b = [&](int j, int s) { return read(at_b + j * 32 * kBlockBytes, s); };
        auto product = [&](v4f (&x)[MT], v4f (&y)[NT]) {
            __builtin_amdgcn_s_setprio(1);     // (before the other wave's fetches and reads)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j)
                    if constexpr (HALVES)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x[i]), __builtin_bit_cast(f16x8, y[j]), acc[i][j], 0, 0, 0);
                    else
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[i]), __builtin_bit_cast(bf16x8, y[j]), acc[i][j], 0, 0, 0);
            __builtin_amdgcn_s_setprio(0);
        };
        if constexpr (ACROSS) {
            // the second parts' 64 bytes are the group beside the first parts': the other one of a pair, whatever the permutation
            const unsigned base = (unsigned)(uintptr_t)(lds_ptr)stage;
            unsigned pa[MT], pb[NT];
#pragma unroll
            for (int i = 0; i < MT; ++i) pa[i] = base + group_a[i];
#pragma unroll
            for (int j = 0; j < NT; ++j) pb[j] = base + group_b[j];
            auto step = [&](auto at) {
                constexpr int kA = 16 * decltype(at)::value * kARow, kB = 16 * decltype(at)::value * kBRow;
                v4f x[MT], y[NT];
                read_turned<kA, 4 * kARow, kB, 4 * kBRow>(x, y, pa, pb);
                if constexpr (HALVES) {
                    v4f xl[MT], yl[NT];
                    unsigned la[MT], lb[NT];
#pragma unroll
                    for (int i = 0; i < MT; ++i) la[i] = pa[i] ^ 64;
#pragma unroll
                    for (int j = 0; j < NT; ++j) lb[j] = pb[j] ^ 64;
                    product(x, y);
                    read_turned<kA, 4 * kARow, kB, 4 * kBRow>(xl, yl, la, lb);
                    product(x, yl);
                    lower(y);
                    product(xl, y);
                } else {
                    product(x, y);
                }
            };
            step(std::integral_constant<int, 0>{});
            step(std::integral_constant<int, 1>{});
            if constexpr (!HALVES) {
                step(std::integral_constant<int, 2>{});
                step(std::integral_constant<int, 3>{});
            }
        } else if constexpr (HALVES) {   // a step's operands are read while the one before it is multiplied
            v4f xh[2][MT], yh[2][NT], xl[2][MT], yl[2][NT];
            auto load = [&](int t, int s) {
#pragma unroll
                for (int i = 0; i < MT; ++i) { xl[t][i] = read_a(i, s + 2); xh[t][i] = read_a(i, s); }
#pragma unroll
                for (int j = 0; j < NT; ++j) { yh[t][j] = read_b(j, s); yl[t][j] = read_b(j, s + 2); }
            };
            load(0, 0);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s == 0) load(1, 1);
                if constexpr (kGradient) {     // (lowered in place: there are no registers for a copy)
                    product(xh[s], yl[s]);
                    product(xh[s], yh[s]);
                    lower(yh[s]);
                    product(xl[s], yh[s]);
                } else {
                    product(xl[s], yh[s]);
                    product(xh[s], yl[s]);
                    product(xh[s], yh[s]);
                }
            }
        } else {
            v4f x[2][MT], y[2][NT];
            auto load = [&](int t, int s) {
#pragma unroll
                for (int i = 0; i < MT; ++i) x[t][i] = read_a(i, s);
#pragma unroll
                for (int j = 0; j < NT; ++j) y[t][j] = read_b(j, s);
            };
            load(0, 0);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                if (s < 3) load((s + 1) & 1, s + 1);
                product(x[s & 1], y[s & 1]);
            }
        }
    };

    if (count > 0) {
        fetch(0, lds_raw);
        for (int b = 0; b < count; ++b) {
            __syncthreads();               // (waits for the wave's own fetches too)
            if (b + 1 < count) fetch(b + 1, lds_raw + ((b + 1) & 1) * kStage);
            multiply(lds_raw + (b & 1) * kStage);
        }
    }

    // ---- results
    Lower f{1.f, 1.f};
    if constexpr (HALVES) {
        const int up = a.a_peak ? raise_of(peak_of(a.a_peak, kPeakGroups), 0) : kDeltaRaise;
        f = lower_by(up + raise_of(peak_of(a.b_peak, kPeakGroups), 0));
    }
    if constexpr (RESULT == kScores) {
        constexpr float kNone = -__builtin_inff();
        const int mw = m0 + 32 * MT * wm + 4 * half, nw = n0 + 32 * NT * wn + row;
        float* const bias_l = reinterpret_cast<float*>(lds_raw);             // [BM]: the biases, minus infinity beyond the last class
        float2* const red = reinterpret_cast<float2*>(lds_raw + BM * 4);     // [WM][BN]
        __syncthreads();
        for (int i = tid; i < BM; i += 64 * kWaves) bias_l[i] = m0 + i < a.M ? (a.bias ? a.bias[m0 + i] : 0.f) : kNone;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int n = nw + 32 * j;
            const bool real = n < a.N;
            int label = real ? a.labels[n] - a.class0 : -1;
            label = label < a.M ? label : -1;
            float top = kNone;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int off = 32 * i + 8 * (r >> 2) + (r & 3);
                    float v = acc[i][j][r];
                    if constexpr (HALVES) v = v * f.first * f.second;
                    // (beyond the last class the operand's rows repeat the last one's, which may be anything)
                    const float b = bias_l[32 * MT * wm + 4 * half + off];
                    v = mw + off < a.M ? v + b : kNone;
                    acc[i][j][r] = v;
                    top = fmaxf(top, v);
                }
            if (a.scores && real) {
                float* to = a.scores + n;
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int m = mw + 32 * i + 8 * (r >> 2) + (r & 3);
                        if (m < a.M) to[(long)m * a.score_row] = acc[i][j][r];
                    }
            }
            const float other = __shfl_xor(top, 32, 64);
            top = fmaxf(top, other);
            const float base = top == kNone ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float v = acc[i][j][r];
                    sum += __builtin_amdgcn_exp2f((v - base) * kLog2e);
                    if (label == mw + 32 * i + 8 * (r >> 2) + (r & 3)) a.label_score[n] = v;
                }
            sum += __shfl_xor(sum, 32, 64);
            if (half == 0) red[wm * BN + 32 * NT * wn + 32 * j + row] = float2{top, sum};
        }
        __syncthreads();
        for (int i = tid; i < BN; i += 64 * kWaves) {
            if (n0 + i >= a.N) continue;
            float2 s = red[i];
#pragma unroll
            for (int w = 1; w < WM; ++w) {
                const float2 o = red[w * BN + i];
                const float top = fmaxf(s.x, o.x), base = top == kNone ? 0.f : top;
                s = float2{top, s.y * __builtin_amdgcn_exp2f((s.x - base) * kLog2e) + o.y * __builtin_amdgcn_exp2f((o.x - base) * kLog2e)};
            }
            a.stats[(long)tm * a.N + n0 + i] = s;
        }
    } else if constexpr (RESULT == kDelta) {
        // By way of LDS as below: a lane has 8 rows of a class
        constexpr int W = 32 * NT, kPitch = W + 4;
        static_assert(W == 64 && (kWaves * 32 * kPitch + BM) * 4 <= 2 * kStage, "a wave's columns are a sum's 64 rows; the ring holds them");
        float* const mine = reinterpret_cast<float*>(lds_raw) + wave * 32 * kPitch;
        float* const bias_l = reinterpret_cast<float*>(lds_raw) + kWaves * 32 * kPitch;
        __syncthreads();
        for (int i = tid; i < BM; i += 64 * kWaves) bias_l[i] = a.bias && m0 + i < a.M ? a.bias[m0 + i] : 0.f;
        const int nw = n0 + W * wn, c = 8 * (lane & 7), n = nw + c;
        float lse[8], weight[8];
        int label[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) {
            const int at = n + z < a.N ? n + z : a.N - 1;
            const float w = a.weight[at];
            lse[z] = a.lse[at];
            weight[z] = n + z < a.N ? w : 0.f;
            label[z] = a.labels[at] - a.class0;
        }
        __syncthreads();
        if (nw >= a.padded) return;                          // (a wave's own places in LDS from here on)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(8 * (r >> 2) + 4 * half + (r & 3)) * kPitch + 32 * j + row] = acc[i][j][r];
            asm volatile("" ::: "memory");
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int of = 8 * q + (lane >> 3), at = 32 * (MT * wm + i) + of, m = m0 + at;
                const v4f lo = *reinterpret_cast<const v4f*>(mine + of * kPitch + c), hi = *reinterpret_cast<const v4f*>(mine + of * kPitch + c + 4);
                v8f v{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                const float bias = bias_l[at];
                float sum = 0.f;
#pragma unroll
                for (int z = 0; z < 8; ++z) {
                    if constexpr (HALVES) v[z] = v[z] * f.first * f.second;
                    const float g = class_delta(v[z] + bias, lse[z], weight[z] != 0.f, label[z] == m);
                    const float weighted = weight[z] != 0.f ? g * weight[z] : 0.f;
                    sum += weighted;
                    v[z] = HALVES ? g * power_of_two(kDeltaRaise) : weighted;
                }
                if (a.db_part) {
                    sum += __shfl_xor(sum, 1, 64);
                    sum += __shfl_xor(sum, 2, 64);
                    sum += __shfl_xor(sum, 4, 64);
                    if ((lane & 7) == 0 && m < a.M) a.db_part[(long)(nw >> 6) * a.M + m] = sum;
                }
                if (!a.delta || m >= a.M) continue;
                char* const to = a.delta + (long)m * a.delta_bytes;
                if constexpr (HALVES) {
                    f16x8 h, l;
#pragma unroll
                    for (int z = 0; z < 8; ++z) {
                        h[z] = (_Float16)v[z];
                        l[z] = (_Float16)((v[z] - (float)h[z]) * kLowUp);
                    }
                    char* const at32 = to + (n >> 5) * kBlockBytes + 2 * (n & 31);
                    *reinterpret_cast<f16x8*>(at32) = h;
                    *reinterpret_cast<f16x8*>(at32 + kBlockBytes / 2) = l;
                } else {
                    *reinterpret_cast<bf16x8*>(to + 2 * n) = __builtin_convertvector(v, bf16x8);
                }
            }
            asm volatile("" ::: "memory");
        }
    } else {
        // A wave's results by way of LDS (a place of its own), 32 rows of 32 NT at a time: whole lines to memory, 8 results a lane
        constexpr int W = 32 * NT, kPitch = W + 4;           // floats; 128-bit words, rows on different banks
        static_assert(kWaves * 32 * kPitch * 4 <= 2 * kStage, "the ring holds them");
        float* const mine = reinterpret_cast<float*>(lds_raw) + wave * 32 * kPitch;
        __syncthreads();                                     // (the last block is read by nobody any more)
        const int nw = n0 + W * wn;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(8 * (r >> 2) + 4 * half + (r & 3)) * kPitch + 32 * j + row] = acc[i][j][r];
            asm volatile("" ::: "memory");                   // (a wave's LDS instructions are served in order)
#pragma unroll
            for (int q = 0; q < W / 16; ++q) {               // 64 lanes: W / 8 a row
                const int of = (64 * q + lane) / (W / 8), c = 8 * ((64 * q + lane) % (W / 8));
                const int m = m0 + 32 * (MT * wm + i) + of, n = nw + c;
                const v4f lo = *reinterpret_cast<const v4f*>(mine + of * kPitch + c), hi = *reinterpret_cast<const v4f*>(mine + of * kPitch + c + 4);
                v8f v{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                if (m >= a.M || n >= a.N) continue;
                const int left = a.N - n;
                if constexpr (RESULT == kPart) {
                    float* const p = a.part + ((long)split * a.M + m) * a.N + n;
                    if (left >= 8) {
                        if (a.add) {
                            const v8f o = load8(p);
#pragma unroll
                            for (int z = 0; z < 8; ++z) v[z] += o[z];
                        }
                        store8(p, v);
                    } else {
#pragma unroll
                        for (int z = 0; z < 8; ++z)
                            if (z < left) p[z] = a.add ? p[z] + v[z] : v[z];
                    }
                } else {
                    float scale = a.row_scale ? a.row_scale[m] : 1.f;
                    scale = a.row_mask && scale != 0.f ? 1.f : scale;
#pragma unroll
                    for (int z = 0; z < 8; ++z) {
                        if constexpr (HALVES) v[z] = v[z] * f.first * f.second;
                        v[z] = scale == 0.f ? 0.f : v[z] * scale;
                    }
                    using T = std::conditional_t<RESULT == kStoreF32, float, bf16>;
                    T* const p = (T*)a.out + (long)m * a.out_row + n;
                    if (left >= 8) {
                        store8(p, v);
                    } else {
#pragma unroll
                        for (int z = 0; z < 8; ++z)
                            if (z < left) store1(p + z, v[z]);
                    }
                }
            }
            asm volatile("" ::: "memory");
        }
    }
}

}  // namespace mpcnn
