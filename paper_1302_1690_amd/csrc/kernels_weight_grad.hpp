// The gradient of a linear layer's weights from rows kept in 8 bits (weight_grad.hip): dw[o][f] = sum over the rows n of dy[n][o] x[n][f].
//
// Products on v_mfma_f32_32x32x16_bf16, sums in fp32.  x in 8 bits times its block's power of two is an exact bf16 number (packed.hpp); bf16 dy is taken as it
// is, fp32 dy as three bf16 parts (24 bits, its exponents as they are; bits below 2^-133, bf16's least, are dropped), whose products are added up, the smallest first: nothing else is rounded but the sums and the result.
//
// A workgroup computes a tile of 32 WM MT x 32 WN NT results, each wave MT x NT of the instruction's.  Both operands have the summed index as the rows of memory;
// blocks of KB rows are fetched into registers while the block before is multiplied, and lie in LDS as they do in memory, as bf16: x is widened on its way
// there, once per workgroup.  The instruction wants 8 rows of one column per lane: ds_read_b64_tr_b16 turns 4 rows x 16 columns around within 16 lanes (lane r
// names 4 columns, r % 4, of row r / 4 and receives column r of all 4).  The 64-byte groups of a row lie permuted by the row's number, on different banks.
//
// Bound by the matrix instruction at the clock that its power leaves, and by what brings x into LDS.  8192 x 4096 x 4096 bf16: e4m3 232-272 us, by the card and by how long it has been at work (290 in a process's first
// calls; 1.01-1.18 PFLOP/s; without x's way into LDS 235 beside 270, a library's plain product 229), int8 264-323 (2.5 instructions a number, e4m3 one half); 13665 x 528 x 4288 fp32 int8 233 us and 19 for the parts' sums, 260 a
// call (238 TFLOP/s), e4m3 219 and 19.  Staged behind the products of a block's middle
// step: 270 us, before its first 300; the fetches of the block after the next have a whole block's products to arrive in.  256 x 256 results on eight waves: half the fetches and a half of the widening of 128 x 128.
#pragma once
#include <type_traits>

#include "packed.hpp"

namespace mpcnn {

struct WeightGradArgs {
    const void* dy;
    long dy_pitch, dy_bytes;               // bytes of all of it, to the last piece's end
    Packed x;
    int N, M, D, padded;                   // rows, outputs, features
    int blocks, per_split, splits;         // along the rows: in all, of a workgroup
    int tiles_m, tiles_n;
    void* dw;                              // [M][D]
    int dw_bf16;
    float* part;                           // [splits][M][D]: partial sums instead
};

typedef __bf16 g_bf16x8 __attribute__((ext_vector_type(8)));
typedef float g_f2 __attribute__((ext_vector_type(2)));
typedef unsigned g_u4 __attribute__((ext_vector_type(4)));

// 8 numbers of packed rows as bf16 (exact).  E4M3: two at a time by the instruction that multiplies with a power of two (whose NaN is not a number's)
template <int KIND>
__device__ __forceinline__ g_bf16x8 widen8(u2 r, unsigned scale)
{
    if constexpr (KIND == MPCNN_I8) return __builtin_convertvector(unpack8(r, scale, KIND), g_bf16x8);
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const float by = scale ? __builtin_bit_cast(float, scale << 23) : 0x1p-127f;
    g_u4 v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        v[2 * h] = __builtin_bit_cast(unsigned, (b2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[h], by, false));
        v[2 * h + 1] = __builtin_bit_cast(unsigned, (b2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(r[h], by, true));
    }
#pragma unroll
    for (int z = 0; z < 4; ++z) v[z] = scale == kNaNScale ? 0x7fc07fc0u : v[z];
    return __builtin_bit_cast(g_bf16x8, v);
}

// The instruction's operands from LDS, of I tiles: 8 rows of one column a lane, at p + K and, the second 4 rows, JUMP bytes on.  (The builtin for
// this waits for all fetches into LDS, also those into the other block's places.)
template <int K, int JUMP>
__device__ __forceinline__ void read_turned(g_bf16x8 (&x)[2], const unsigned (&p)[2])
{
    g_f2 a0, a1, b0, b1;
    asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\t"
                 "ds_read_b64_tr_b16 %2, %5 offset:%6\n\tds_read_b64_tr_b16 %3, %5 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1)
                 : "v"(p[0]), "v"(p[1]), "n"(K), "n"(K + JUMP)
                 : "memory");
    x[0] = __builtin_bit_cast(g_bf16x8, v4f{a0[0], a0[1], a1[0], a1[1]});
    x[1] = __builtin_bit_cast(g_bf16x8, v4f{b0[0], b0[1], b1[0], b1[1]});
}
template <int K, int JUMP>
__device__ __forceinline__ void read_turned(g_bf16x8 (&x)[4], const unsigned (&p)[4])
{
    g_f2 a0, a1, b0, b1, c0, c1, d0, d1;
    asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %2, %9 offset:%12\n\tds_read_b64_tr_b16 %3, %9 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                 "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1), "=&v"(c0), "=&v"(c1), "=&v"(d0), "=&v"(d1)
                 : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(K), "n"(K + JUMP)
                 : "memory");
    x[0] = __builtin_bit_cast(g_bf16x8, v4f{a0[0], a0[1], a1[0], a1[1]});
    x[1] = __builtin_bit_cast(g_bf16x8, v4f{b0[0], b0[1], b1[0], b1[1]});
    x[2] = __builtin_bit_cast(g_bf16x8, v4f{c0[0], c0[1], c1[0], c1[1]});
    x[3] = __builtin_bit_cast(g_bf16x8, v4f{d0[0], d0[1], d1[0], d1[1]});
}

// DIRECT (bf16 dy in aligned rows of whole 16-byte pieces): dy's blocks go from memory straight into LDS
template <typename T, int KIND, int WM, int WN, int MT, int NT, int KB, bool DIRECT>
__global__ __launch_bounds__(64 * WM * WN) void weight_grad_kernel(WeightGradArgs a)
{
    constexpr int BM = 32 * WM * MT, BN = 32 * WN * NT, kThreads = 64 * WM * WN, S = KB / 16;
    constexpr int P = sizeof(T) == 4 ? 3 : 1;            // parts of dy
    constexpr int kARow = 2 * BM, kBRow = 2 * BN;        // bytes
    constexpr int kPart = KB * kARow, kStage = P * kPart + KB * kBRow;
    constexpr int AI = KB * BM / 8 / kThreads, BI = KB * BN / 16 / kThreads;
    static_assert(AI * 8 * kThreads == KB * BM && BI * 16 * kThreads == KB * BN, "the threads share a block evenly");
    static_assert(!DIRECT || P == 1, "as it lies in memory");
    extern __shared__ __attribute__((aligned(256))) char lds_raw[];
    typedef __attribute__((address_space(3))) void* lds_ptr;
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

    // ---- blocks from memory: dy a piece of 8 numbers of AI rows, x 16 numbers of BI rows a thread
    Raw8<T> ra[DIRECT ? 1 : AI];
    g_u4 rb[BI];
    unsigned rs[BI];
    unsigned va[DIRECT ? AI : 1];                        // DIRECT: the pieces' places in memory, for their places in LDS
    if constexpr (DIRECT)
#pragma unroll
        for (int i = 0; i < AI; ++i) {
            const unsigned at = (unsigned)((wave * AI + i) * 1024 + 16 * lane), k = at / kARow;
            va[i] = k * (unsigned)(2 * a.dy_pitch) + 16u * ((at % kARow / 16) ^ 4 * (k & 3));
        }
    // (from a block's first row on, with the matrix's end as its bound: rows beyond the last come as zeros)
    auto from = [&](const void* m, long offset, long bytes) {
        const long left = bytes - offset;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>((const char*)m + (left > 0 ? offset : 0)), 0,
                                                 left <= 0 ? 0 : left < 0x7fffffff ? (int)left : 0x7fffffff, 0x00020000);
    };
    auto fetch_direct = [&](int block, char* to) {
        if constexpr (DIRECT) {
            const __amdgpu_buffer_rsrc_t dy = from(a.dy, ((long)(first + block) * KB * a.dy_pitch + m0) * 2, a.dy_bytes);
#pragma unroll
            for (int i = 0; i < AI; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(dy, (lds_ptr)(to + (wave * AI + i) * 1024), 16, (int)va[i], 0, 0, 0);
        }
    };
    auto fetch = [&](int block) {
        const long k0 = (long)(first + block) * KB;
        // (a row behind each of the block's: 8 numbers from its last piece on are the matrix's, and what is beyond its columns is dropped)
        const bool inside = k0 + KB < a.N && a.M >= 8;
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < AI; ++i) {
                const int q = tid + kThreads * i, k = q / (BM / 8), at = m0 + 8 * (q % (BM / 8));
                if (inside) ra[i] = raw8((const T*)a.dy + (k0 + k) * a.dy_pitch + (at < a.M ? at : 0));
                else if (k0 + k < a.N && at < a.M) ra[i] = raw8_of((const T*)a.dy + (k0 + k) * a.dy_pitch, at, a.M);
                else ra[i] = Raw8<T>{};
            }
#pragma unroll
        for (int i = 0; i < BI; ++i) {                   // (always as many loads as kLoads.  Rows beyond the last: the last one, times zeros of dy; columns: dropped)
            const int q = tid + kThreads * i, at = n0 + 16 * (q % (BN / 16));
            const long k = k0 + q / (BN / 16), kc = k < a.N ? k : a.N - 1;
            const int ac = at < a.padded ? at : a.padded - 16;
            rb[i] = *reinterpret_cast<const g_u4*>(a.x.values + kc * a.padded + ac);
            rs[i] = a.x.scales[kc * (a.padded / kBlock) + ac / kBlock];
        }
    };
    constexpr int kLoads = 2 * BI;
    // ---- and into LDS.  (By hand: the compiler would wait for the direct fetches before each of its own writes.)
    auto write = [&](const char* at, g_bf16x8 v) {
        asm volatile("ds_write_b128 %0, %1" ::"v"((unsigned)(uintptr_t)(lds_ptr)at), "v"(v) : "memory");
    };
    auto stage = [&](char* to) {
#pragma unroll
        for (int i = 0; i < BI; ++i) asm volatile("" : "+v"(rb[i]), "+v"(rs[i]));        // (nothing of it earlier: it would wait)
        if constexpr (!DIRECT)
#pragma unroll
            for (int i = 0; i < AI; ++i) {
                const int q = tid + kThreads * i, k = q / (BM / 8), p = q % (BM / 8);
                char* const at = to + k * kARow + 16 * (p ^ 4 * (k & 3));
                if constexpr (P == 1) {
                    write(at, __builtin_bit_cast(g_bf16x8, ra[i].a));
                } else {
                    v8f v = widen(ra[i]);
#pragma unroll
                    for (int z = 0; z < P; ++z) {
                        g_u4 h;                          // (cut off, not rounded: 8 bits of the 24 each, and the largest numbers do not become infinite)
#pragma unroll
                        for (int q = 0; q < 4; ++q) h[q] = __builtin_amdgcn_perm(bits_of(v[2 * q + 1]), bits_of(v[2 * q]), 0x07060302);
                        write(at + z * kPart, __builtin_bit_cast(g_bf16x8, h));
#pragma unroll
                        for (int q = 0; q < 8; ++q) v[q] -= __builtin_bit_cast(float, bits_of(v[q]) & 0xffff0000u);
                    }
                }
            }
#pragma unroll
        for (int h = 0; h < 2 * BI; ++h) {
            const int i = h / 2, q = tid + kThreads * i, k = q / (BN / 16), p = 2 * (q % (BN / 16)) + h % 2;
            write(to + P * kPart + k * kBRow + 16 * (p ^ 4 * (k & 3)), widen8<KIND>(u2{rb[i][2 * (h % 2)], rb[i][2 * (h % 2) + 1]}, rs[i]));
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
    unsigned at_a[MT], at_b[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) at_a[i] = (unsigned)(uintptr_t)(lds_ptr)lds_raw + of_row * kARow + of_col + 64 * ((MT * wm + i) ^ turn);
#pragma unroll
    for (int j = 0; j < NT; ++j) at_b[j] = (unsigned)(uintptr_t)(lds_ptr)lds_raw + P * kPart + of_row * kBRow + of_col + 64 * ((NT * wn + j) ^ turn);

    // A block's products; the next block goes into LDS beside the first of them, and the one after is fetched then
    auto work = [&](int b) {
        const unsigned now = (unsigned)(b & 1) * kStage;
        char* const next = lds_raw + kStage - now;
        unsigned pa[MT], pb[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) pa[i] = at_a[i] + now;
#pragma unroll
        for (int j = 0; j < NT; ++j) pb[j] = at_b[j] + now;
        fetch_direct(b + 1 < count ? b + 1 : b, next);   // (beyond the last block the last one again, for nobody: no branch keeps the compiler from its schedule)
        auto step = [&](auto at) {
            constexpr int s = decltype(at)::value;
            g_bf16x8 x[MT], y[NT];
            read_turned<16 * s * kBRow, 4 * kBRow>(y, pb);
            auto part = [&](auto which) {
                constexpr int z = decltype(which)::value;
                read_turned<z * kPart + 16 * s * kARow, 4 * kARow>(x, pa);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y[j], acc[i][j], 0, 0, 0);
            };
            if constexpr (P == 3) {                      // (the smallest first)
                part(std::integral_constant<int, 2>{});
                part(std::integral_constant<int, 1>{});
            }
            part(std::integral_constant<int, 0>{});
            if constexpr (s == S / 2) {
                stage(next);
                fetch(b + 2 < count ? b + 2 : count - 1);
            }
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        if constexpr (S > 2) {
            step(std::integral_constant<int, 2>{});
            step(std::integral_constant<int, 3>{});
        }
    };
    // Everybody's writes into LDS are done, those of the direct fetches too, but not the loads of the block after the next (a barrier of the compiler's would
    // wait for them)
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    auto meet_all = [&](auto on_the_way) {
        if constexpr (!DIRECT) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(on_the_way)::value ? kLoads : 0) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (count > 0) {
        fetch_direct(0, lds_raw);
        fetch(0);
        stage(lds_raw);
        fetch(count > 1 ? 1 : 0);
        for (int b = 0; b < count; ++b) {
            meet_all(yes);
            work(b);
        }
    }

    // ---- results by way of LDS, a wave's place its own, 32 rows of 32 NT at a time: whole lines to memory, 8 results a lane
    constexpr int W = 32 * NT, kPitch = W + 4;           // floats; 128-bit words, rows on different banks
    static_assert(WM * WN * 32 * kPitch * 4 <= 2 * kStage, "the blocks' places hold them");
    float* const mine = reinterpret_cast<float*>(lds_raw) + wave * 32 * kPitch;
    meet_all(no);                                     // (the last block is read by nobody any more)
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
            const int m = m0 + 32 * (MT * wm + i) + of, n = n0 + W * wn + c;
            const v4f lo = *reinterpret_cast<const v4f*>(mine + of * kPitch + c), hi = *reinterpret_cast<const v4f*>(mine + of * kPitch + c + 4);
            const v8f v{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (m >= a.M || n >= a.D) continue;
            const long at = (long)m * a.D;
            if (a.part) store8_of(a.part + (long)split * a.M * a.D + at, n, a.D, v);
            else if (a.dw_bf16) store8_of((bf16*)a.dw + at, n, a.D, v);
            else store8_of((float*)a.dw + at, n, a.D, v);
        }
        asm volatile("" ::: "memory");
    }
}

// bf16 dy into aligned rows of whole 16-byte pieces [N][to_pitch], zeros behind its columns: a piece a thread
__global__ __launch_bounds__(256) void weight_grad_align_kernel(const bf16* dy, long pitch, long N, int M, bf16* to, int to_pitch)
{
    const unsigned pieces = (unsigned)to_pitch / 8;
    const long all = N * pieces;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long)gridDim.x * 256) {
        const long n = all <= 0xffffffffl ? (long)((unsigned)i / pieces) : i / pieces;
        const int at = 8 * (int)(i - n * pieces);
        const bf16* const row = dy + n * pitch;
        const v8f v = at + 8 <= M ? widen(odd8(row + at), row) : load8_of(row, at, M);
        *reinterpret_cast<g_bf16x8*>(to + n * to_pitch + at) = __builtin_convertvector(v, g_bf16x8);
    }
}

// The splits' sums (without splits, zeros): 64 numbers a workgroup at a time, a wave every fourth split, eight on their way at once; the waves' sums in their order
__global__ __launch_bounds__(256) void weight_grad_sum_kernel(const float* part, int splits, long n, void* out, int out_bf16)
{
    __shared__ float red[2][3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int flip = 0;
    for (long base = 64 * (long)blockIdx.x; base < n; base += 64 * (long)gridDim.x, flip ^= 1) {
        const long i = base + lane;
        float s = 0.f;
        if (i < n) {
            int z = wave;
            for (; z + 28 < splits; z += 32) {
                float v[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] = part[(long)(z + 4 * q) * n + i];
#pragma unroll
                for (int q = 0; q < 8; ++q) s += v[q];
            }
#pragma unroll 4
            for (; z < splits; z += 4) s += part[(long)z * n + i];
        }
        if (wave) red[flip][wave - 1][lane] = s;
        __syncthreads();
        if (wave || i >= n) continue;
        s = ((s + red[flip][0][lane]) + red[flip][1][lane]) + red[flip][2][lane];
        if (out_bf16) ((bf16*)out)[i] = (bf16)s;
        else ((float*)out)[i] = s;
    }
}

}  // namespace mpcnn
