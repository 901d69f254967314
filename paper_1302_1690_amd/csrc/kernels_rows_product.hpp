// The matrix product of the class layer on rows of features (class_rows.hip): C[m][n] = sum_k A[m][k] B[n][k], both operands with k
// running fastest, 16-bit numbers on v_mfma_f32_32x32x16, sums in fp32.
//
// Operands.  bf16 storage: as they are.  fp32 storage: two fp16 parts per number (x 2^e = h + l, ranges.hpp), which lie in turn,
// 32 numbers' first parts and their second parts, so that one 128-byte block of a row is 64 bf16 numbers or 32 fp32 ones and the kernel's
// fetches are the same; the products are h h', h l' and l h' (what is left out, l l', is below 2^-22 of a product).  k is padded with
// zeros to whole blocks; rows beyond the last are not read (the last one is, again, and its results dropped).
//
// A workgroup computes a tile of 32 WM MT x 32 WN NT results, each wave MT x NT of the instruction's, in accumulators.  Both operands' next
// blocks come from memory straight into the LDS buffer that is not being multiplied (128 bits per lane, a barrier per block).  An LDS row is a
// block (128 bytes); its 16-byte pieces lie permuted by half the row's number (two rows are the 256 bytes of the banks), so that the lanes of an
// operand's fetch, which read one piece each of 32 rows, find them on different banks.  The permutation is made by the addresses in memory that the lanes fetch from.
//
// Results: the classes' scores with their bias (m = class, n = row), of which only each row's largest and sum of exponentials over the
// tile's classes leave the kernel (and the score of its label), or which are stored too; or products, stored rounded; or partial sums.
#pragma once
#include <type_traits>

#include "any_address.hpp"
#include "ranges.hpp"

namespace mpcnn {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kBlockBytes = 128;           // of a row of an operand
constexpr float kLog2e = 1.4426950408889634f;

struct ProductArgs {
    const char *A, *B;                     // rows of blocks
    long a_row, b_row;                     // bytes
    int M, N;
    int blocks, per_split;                 // along k: in all, of a workgroup
    int tiles_m, tiles_n, splits;
    const unsigned *a_peak, *b_peak;       // fp32 storage: what the operands were raised by (null: by a_up, b_up)
    int a_words, b_words, a_up, b_up;
    // scores
    const float* bias;                     // [M] or null
    const int* labels;                     // [N]
    float2* stats;                         // [tiles_m][N]: largest, sum of exp(score - largest)
    float* label_score;                    // [N]
    float* scores;                         // [M][score_row], or null
    long score_row;
    int class0;                            // the first class of A
    // products
    void* out;                             // [M][out_row]
    long out_row;
    const float* row_scale;                // [M], or null
    float* part;                           // [splits][M][N]: partial sums instead (added to what is there: add)
    int add;
};
enum { kScores = 0, kStoreF32 = 1, kStoreBf16 = 2, kPart = 3 };

__device__ __forceinline__ int raised_by(const unsigned* peak, int words, int up)
{
    return peak ? raise_of(peak_of(peak, words), 0) : up;
}

template <int WM, int WN, int MT, int NT, bool HALVES, int RESULT>
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

    // ---- fetches: rows 8 q .. 8 q + 7 of a block, lane l the piece l % 8 of row 8 q + l / 8 as it lies in LDS
    typedef __attribute__((address_space(3))) void* lds_ptr;
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
        const int r = 8 * (wave * AI + i) + (lane >> 3), left = a.M - 1 - m0;
        va[i] = (unsigned)(r < left ? r : left) * (unsigned)a.a_row + piece[i & 1];
    }
#pragma unroll
    for (int i = 0; i < BI; ++i) {
        const int r = 8 * (wave * BI + i) + (lane >> 3), left = a.N - 1 - n0;
        vb[i] = (unsigned)(r < left ? r : left) * (unsigned)a.b_row + piece[i & 1];
    }
    auto fetch = [&](int block, char* stage) {
#pragma unroll
        for (int i = 0; i < AI; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(stage + (wave * AI + i) * 1024), 16, (int)va[i], block * kBlockBytes, 0, 0);
#pragma unroll
        for (int i = 0; i < BI; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(stage + BM * kBlockBytes + (wave * BI + i) * 1024), 16, (int)vb[i],
                                                     block * kBlockBytes, 0, 0);
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
    auto multiply = [&](const char* stage) {
        auto read = [&](int at, int s) { return *reinterpret_cast<const v4f*>(stage + at + 16 * ((2 * s + half) ^ mix)); };
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
        // a step's operands are read while the one before it is multiplied
        if constexpr (HALVES) {
            v4f xh[2][MT], yh[2][NT], xl[2][MT], yl[2][NT];
            auto load = [&](int t, int s) {
#pragma unroll
                for (int i = 0; i < MT; ++i) { xl[t][i] = read(at_a + i * 32 * kBlockBytes, s + 2); xh[t][i] = read(at_a + i * 32 * kBlockBytes, s); }
#pragma unroll
                for (int j = 0; j < NT; ++j) { yh[t][j] = read(at_b + j * 32 * kBlockBytes, s); yl[t][j] = read(at_b + j * 32 * kBlockBytes, s + 2); }
            };
            load(0, 0);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s == 0) load(1, 1);
                product(xl[s], yh[s]);
                product(xh[s], yl[s]);
                product(xh[s], yh[s]);
            }
        } else {
            v4f x[2][MT], y[2][NT];
            auto load = [&](int t, int s) {
#pragma unroll
                for (int i = 0; i < MT; ++i) x[t][i] = read(at_a + i * 32 * kBlockBytes, s);
#pragma unroll
                for (int j = 0; j < NT; ++j) y[t][j] = read(at_b + j * 32 * kBlockBytes, s);
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
        const int up = raised_by(a.a_peak, a.a_words, a.a_up) + raised_by(a.b_peak, a.b_words, a.b_up);
        f = lower_by(up);
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
            int label = real && a.stats ? a.labels[n] - a.class0 : -1;
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
            if (!a.stats) continue;
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
        if (!a.stats) return;
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
                    const float scale = a.row_scale ? a.row_scale[m] : 1.f;   // (0: nothing of the row, whatever it is multiplied with)
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
