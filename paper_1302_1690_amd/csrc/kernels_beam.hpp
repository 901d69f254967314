// Beam search over many classes: which continuations go on (beam.hip), and the states that follow them.
//
//   s[k][v] = score + bias (fp32; a class whose bias is minus infinity is off),  lse[k] = log sum over v of exp s[k][v],
//   value(k, v) = total[k] + (s[k][v] - lse[k]) in 64 bits;  the `width` largest of a sequence's beams x classes, ties to the lowest beam, then class.
// A finished beam offers one candidate, the class that ends a sequence, at its total; a dead one (total minus infinity) none.
//
// Two launches.  The first goes through the scores once and is bound by memory: a wave takes chunks of 1024 classes and leaves each chunk's largest score; a workgroup
// leaves its classes' largest and sum of exponentials.  The second, a workgroup per sequence, joins the sums and reads again only what can matter: the chunks whose
// largest are among the `width` best of all.  (Let an element of another chunk be among the best: `width` chunks have a largest that is better, and so is
// not below it, and these are as many elements that come before it.)  Order is by (value, then place), which no two candidates share, so the
// result does not depend on timing.  lse is a sum of fp32 exponentials, joined in 64 bits: within one beam the order is the scores', exactly.
#pragma once
#include <type_traits>

#include "any_address.hpp"
#include "lanes.hpp"

namespace mpcnn {

constexpr int kChunk = 1024;               // classes
constexpr int kMaxBeams = 64;
constexpr int kPickThreads = 512, kPickWaves = kPickThreads / 64;

struct BeamArgs {
    const void* scores;
    long pitch;                            // of a row, or of a class (BeamColumn)
    const float* bias;
    const float* totals;
    const unsigned char* done;             // null: none
    int end;
    int sequences, beams, width;
    int V, chunks, parts, part_chunks;     // chunks of a row, workgroups of a row, chunks of a workgroup
    float2* stats;                         // [rows][parts]
    float* tops;                           // [rows][chunks]
    float* totals_out;
    int *parents, *classes;
    unsigned char* done_out;
};

// A row's chunks: a lane has E numbers (16 bytes) of each J stretches.  The classes' shares do not depend on where the row lies, so rows that hold the same have
// the same sums (and beams that are alike are equals).
template <typename T>
struct BeamRow {
    static constexpr int E = 16 / sizeof(T), J = kChunk / (64 * E);
    using Block = std::conditional_t<sizeof(T) == 2, Odd8, Raw<float, 4>>;
    const T* from;
    int V;
    bool odd;                              // begins between two words (bf16)
    const float* bias;
    __device__ BeamRow(const BeamArgs& a, long row) : from((const T*)a.scores + row * a.pitch), V(a.V), odd((uintptr_t)from & 2), bias(a.bias) {}
    __device__ static int number(int j) { return E * ((int)(threadIdx.x & 63) + 64 * j); }
    __device__ void fetch(int chunk, Block (&u)[J]) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = kChunk * chunk + number(j);
            if (at >= V) continue;
            if constexpr (sizeof(T) == 4) u[j] = raw_of<4>(from, at, V);
            else if (at + 8 > V) u[j] = odd8_of(from, at, V);
            else if (odd) u[j] = odd8(from + at);
            else u[j].a = *reinterpret_cast<const Odd8::u4_any*>(from + at);
        }
    }
    // scores with the bias; minus infinity beyond the row and for classes that are off, whatever is there
    __device__ void scores(int chunk, const Block (&u)[J], float (&s)[J][E]) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = kChunk * chunk + number(j);
            float b[E];
            if (bias && at + E <= V) {
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const f4_any w = *reinterpret_cast<const f4_any*>(bias + at + e);
#pragma unroll
                    for (int z = 0; z < 4; ++z) b[e + z] = w[z];
                }
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) b[e] = bias && at + e < V ? bias[at + e] : 0.f;
            }
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int e = 0; e < E; ++e) s[j][e] = u[j].a[e];
            } else {
                const v8f v = widen(u[j], from);
#pragma unroll
                for (int e = 0; e < E; ++e) s[j][e] = v[e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) s[j][e] = at + e < V && b[e] != -__builtin_inff() ? s[j][e] + b[e] : -__builtin_inff();
        }
    }
};

// The same of scores that lie [class][row], fp32, as a class layer leaves them, with their bias
struct BeamColumn {
    static constexpr int E = 4, J = kChunk / (64 * E);
    typedef float Block[E];
    const float* from;
    long pitch;
    int V;
    __device__ BeamColumn(const BeamArgs& a, long row) : from((const float*)a.scores + row), pitch(a.pitch), V(a.V) {}
    __device__ static int number(int j) { return E * ((int)(threadIdx.x & 63) + 64 * j); }
    __device__ void fetch(int chunk, Block (&u)[J]) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int at = kChunk * chunk + number(j) + e;
                u[j][e] = at < V ? from[at * pitch] : -__builtin_inff();
            }
    }
    __device__ void scores(int, const Block (&u)[J], float (&s)[J][E]) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) s[j][e] = u[j][e];
    }
};

__device__ __forceinline__ bool beam_goes_on(const BeamArgs& a, long row)
{
    return a.totals[row] > -__builtin_inff() && !(a.done && a.done[row]);     // (a NaN does not)
}

// exp(x - top) for x <= top; 0 for minus infinity
__device__ __forceinline__ float exp_below(float x, float top) { return __builtin_amdgcn_exp2f((x - top) * 1.4426950408889634f); }

__device__ __forceinline__ float largest64(float m)
{
#pragma unroll
    for (int i = 1; i < 64; i *= 2) m = fmaxf(m, __shfl_xor(m, i, 64));
    return m;
}

template <typename T>
__global__ __launch_bounds__(256) void beam_stats_kernel(BeamArgs a)
{
    using Row = BeamRow<T>;
    __shared__ float2 red[4];
    const long row = blockIdx.x / a.parts;
    const int part = (int)(blockIdx.x % a.parts), lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (!beam_goes_on(a, row)) return;
    const Row r(a, row);
    const int end = (part + 1) * a.part_chunks < a.chunks ? (part + 1) * a.part_chunks : a.chunks;
    int c = part * a.part_chunks + wave;
    typename Row::Block u[Row::J];
    if (c < end) r.fetch(c, u);
    float top = -__builtin_inff(), sum = 0.f;
    for (; c < end; c += 4) {
        float s[Row::J][Row::E];
        r.scores(c, u, s);
        if (c + 4 < end) r.fetch(c + 4, u);
        float most = s[0][0];
#pragma unroll
        for (int j = 0; j < Row::J; ++j)
#pragma unroll
            for (int e = 0; e < Row::E; ++e) most = fmaxf(most, s[j][e]);
        most = largest64(most);
        if (lane == 0) a.tops[row * a.chunks + c] = most;
        const float now = fmaxf(top, most), base = now == -__builtin_inff() ? 0.f : now;
        sum *= exp_below(top, base);
        top = now;
#pragma unroll
        for (int j = 0; j < Row::J; ++j)
#pragma unroll
            for (int e = 0; e < Row::E; ++e) sum += exp_below(s[j][e], base);
    }
    sum = sum64(sum);
    if (lane == 0) red[wave] = float2{top, sum};
    __syncthreads();
    if (threadIdx.x == 0) {
        float2 all = red[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) {
            const float now = fmaxf(all.x, red[w].x), base = now == -__builtin_inff() ? 0.f : now;
            all = float2{now, all.y * exp_below(all.x, base) + red[w].y * exp_below(red[w].x, base)};
        }
        a.stats[row * a.parts + part] = all;
    }
}

// Scores [class][row]: a workgroup has a chunk of classes of four rows, a thread four classes
__global__ __launch_bounds__(256) void beam_columns_kernel(BeamArgs a)
{
    __shared__ float tops[4][4], sums[4][4];
    const int chunk = (int)(blockIdx.x % a.chunks), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long row0 = 4 * (long)(blockIdx.x / a.chunks), rows = (long)a.sequences * a.beams;
    v4f s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int at = kChunk * chunk + 256 * i + (int)threadIdx.x;
        s[i] = at < a.V ? *reinterpret_cast<const v4f*>((const float*)a.scores + at * a.pitch + row0) : v4f(-__builtin_inff());
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float m = largest64(fmaxf(fmaxf(s[0][r], s[1][r]), fmaxf(s[2][r], s[3][r])));
        if (lane == 0) tops[wave][r] = m;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float top = fmaxf(fmaxf(tops[0][r], tops[1][r]), fmaxf(tops[2][r], tops[3][r])), base = top == -__builtin_inff() ? 0.f : top;
        const float sum = sum64((exp_below(s[0][r], base) + exp_below(s[1][r], base)) + (exp_below(s[2][r], base) + exp_below(s[3][r], base)));
        if (lane == 0) sums[wave][r] = sum;
    }
    __syncthreads();
    const int r = threadIdx.x;
    if (r >= 4 || row0 + r >= rows) return;
    const float top = fmaxf(fmaxf(tops[0][r], tops[1][r]), fmaxf(tops[2][r], tops[3][r]));
    a.tops[(row0 + r) * a.chunks + chunk] = top;
    a.stats[(row0 + r) * a.parts + chunk] = float2{top, (sums[0][r] + sums[1][r]) + (sums[2][r] + sums[3][r])};
}

// ---- the second launch

typedef unsigned long long u64;
// Values in an order of whole numbers; 0: no candidate
__device__ __forceinline__ u64 key_of(double v)
{
    if (!(v > -__builtin_inf())) return 0;
    const u64 b = __builtin_bit_cast(u64, v);
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double value_of(u64 key) { return __builtin_bit_cast(double, key >> 63 ? key ^ 1ull << 63 : ~key); }
__device__ __forceinline__ u64 largest64(u64 k)
{
#pragma unroll
    for (int i = 1; i < 64; i *= 2) {
        const u64 o = __shfl_xor(k, i, 64);
        k = o > k ? o : k;
    }
    return k;
}

// The best of the wave's candidates and where it is (all lanes' places differ): the lowest place of the largest key
__device__ __forceinline__ u64 best_of(u64 key, unsigned place, unsigned* best)
{
    const u64 top = largest64(key);
    u64 lanes = __ballot(key == top);
    unsigned p = 0xffffffffu;
    while (lanes) {                        // (one, but for ties)
        const int l = __builtin_ctzll(lanes);
        const unsigned o = (unsigned)__builtin_amdgcn_readlane((int)place, l);
        p = o < p ? o : p;
        lanes &= lanes - 1;
    }
    *best = p;
    return top;
}

struct BeamOffer { u64 key; unsigned place; };   // of a chunk: beam * chunks + chunk; of a candidate: chosen chunk << 10 | number

template <typename Row>
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(BeamArgs a)
{
    constexpr int R = 4;                   // chunks of a lane at once
    extern __shared__ __attribute__((aligned(16))) char lds_raw[];
    __shared__ double lse[kMaxBeams];
    __shared__ float total[kMaxBeams];
    __shared__ unsigned char kind[kMaxBeams];            // 0: offers nothing, 1: goes on, 2: finished
    __shared__ u64 part_key[kPickWaves * kMaxBeams];
    __shared__ unsigned part_place[kPickWaves * kMaxBeams];
    __shared__ u64 chosen_key[kMaxBeams];
    __shared__ unsigned chosen_place[kMaxBeams];
    __shared__ unsigned count;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int W = a.width, K = a.beams;
    u64* const cand_key = reinterpret_cast<u64*>(lds_raw);             // [W W]
    unsigned* const cand_place = reinterpret_cast<unsigned*>(lds_raw + sizeof(u64) * W * W);
    const long row0 = (long)blockIdx.x * K;

    // ---- the beams' sums
    for (int k = wave; k < K; k += kPickWaves) {
        const long row = row0 + k;
        const float t = a.totals[row];
        int is = t > -__builtin_inff() ? (a.done && a.done[row] ? 2 : 1) : 0;
        double l = 0.0;
        if (is == 1) {
            float top = -__builtin_inff();
            for (int p = lane; p < a.parts; p += 64) top = fmaxf(top, a.stats[row * a.parts + p].x);
            top = largest64(top);
            double sum = 0.0;
            for (int p = lane; p < a.parts; p += 64) {
                const float2 s = a.stats[row * a.parts + p];
                if (s.x > -__builtin_inff() || s.y != 0.f) sum += (double)s.y * exp((double)s.x - (double)top);
            }
#pragma unroll
            for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i, 64);
            l = (double)top + log(sum);
            if (!(l > -__builtin_inf() && l < __builtin_inf())) is = 0;        // nothing is on, or a score is not finite
        }
        if (lane == 0) { lse[k] = l; total[k] = t; kind[k] = (unsigned char)is; }
    }
    if (tid < W) { chosen_key[tid] = 0; chosen_place[tid] = 0; }
    if (tid == 0) count = 0;
    __syncthreads();

    // ---- each wave's best chunks: winners so far (slot 0, winner i in lane i) against the next R of every lane
    const int all = K * a.chunks;          // (below 2^28)
    u64 won_key = 0;
    unsigned won_place = 0xffffffffu;
    for (int base = wave * 64 * R; base < all; base += kPickThreads * R) {
        u64 key[R + 1];
        unsigned place[R + 1];
        key[R] = won_key; place[R] = won_place;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = base + 64 * r + lane;
            key[r] = 0; place[r] = (unsigned)i;
            if (i >= all) continue;
            const int k = i / a.chunks, c = i - k * a.chunks;
            if (kind[k] == 1) key[r] = key_of((double)total[k] + ((double)a.tops[(row0 + k) * a.chunks + c] - lse[k]));
            else if (kind[k] == 2 && c == 0) key[r] = key_of((double)total[k]);       // (its only candidate: see below)
        }
        won_key = 0; won_place = 0xffffffffu;
        for (int w = 0; w < W; ++w) {
            u64 mine = key[0];
            unsigned at = place[0];
#pragma unroll
            for (int r = 1; r <= R; ++r)
                if (key[r] > mine || (key[r] == mine && place[r] < at)) { mine = key[r]; at = place[r]; }
            unsigned best;
            const u64 top = best_of(mine, at, &best);
            if (!top) break;
#pragma unroll
            for (int r = 0; r <= R; ++r)
                if (key[r] == top && place[r] == best) key[r] = 0;
            if (lane == w) { won_key = top; won_place = best; }
        }
    }
    if (lane < W) { part_key[wave * W + lane] = won_key; part_place[wave * W + lane] = won_place; }
    __syncthreads();

    // ---- the best chunks of all waves, by how many come before each
    auto before = [](u64 k, unsigned p, u64 key, unsigned place) { return k > key || (k == key && p < place); };
    for (int i = tid; i < kPickWaves * W; i += kPickThreads) {
        const u64 key = part_key[i];
        if (!key) continue;
        const unsigned place = part_place[i];
        int rank = 0;
        for (int o = 0; o < kPickWaves * W; ++o) rank += before(part_key[o], part_place[o], key, place);
        if (rank < W) { chosen_key[rank] = key; chosen_place[rank] = place; }
    }
    __syncthreads();

    // ---- their numbers that are not below the last chosen chunk's largest, at most W of each
    const u64 least = chosen_key[W - 1];
    auto offer = [&](u64 key, unsigned place) {
        const unsigned i = atomicAdd(&count, 1u);
        cand_key[i] = key;
        cand_place[i] = place;
    };
    for (int w = wave; w < W; w += kPickWaves) {
        if (!chosen_key[w]) continue;
        const int k = (int)chosen_place[w] / a.chunks, c = (int)chosen_place[w] - k * a.chunks;
        if (kind[k] == 2) {
            if (lane == 0) offer(chosen_key[w], (unsigned)w << 10);
            continue;
        }
        const Row r(a, row0 + k);
        typename Row::Block u[Row::J];
        r.fetch(c, u);
        float s[Row::J][Row::E];
        r.scores(c, u, s);
        u64 key[Row::J][Row::E];
#pragma unroll
        for (int j = 0; j < Row::J; ++j)
#pragma unroll
            for (int e = 0; e < Row::E; ++e) {
                const u64 v = key_of((double)total[k] + ((double)s[j][e] - lse[k]));
                key[j][e] = v >= least ? v : 0;
            }
        for (int n = 0; n < W; ++n) {
            u64 mine = 0;
            unsigned at = 0xffffffffu;
#pragma unroll
            for (int j = 0; j < Row::J; ++j)
#pragma unroll
                for (int e = 0; e < Row::E; ++e)
                    if (key[j][e] > mine) { mine = key[j][e]; at = (unsigned)(Row::number(j) + e); }       // (the lowest number of equals)
            unsigned best;
            const u64 top = best_of(mine, at, &best);
            if (!top) break;
#pragma unroll
            for (int j = 0; j < Row::J; ++j)
#pragma unroll
                for (int e = 0; e < Row::E; ++e)
                    if (best == (unsigned)(Row::number(j) + e)) key[j][e] = 0;
            if (lane == 0) offer(top, (unsigned)w << 10 | best);
        }
    }
    __syncthreads();

    // ---- the best of these
    const int n = (int)count;
    const long out = (long)blockIdx.x * W;
    auto place_of = [&](unsigned p) -> u64 {
        const unsigned chunk = chosen_place[p >> 10];
        const int k = (int)chunk / a.chunks, c = (int)chunk - k * a.chunks;
        if (kind[k] == 2) return (u64)k * (unsigned)a.V + (unsigned)a.end;
        return (u64)k * (unsigned)a.V + (unsigned)(kChunk * c + (int)(p & (kChunk - 1)));
    };
    for (int i = tid; i < n; i += kPickThreads) {
        const u64 key = cand_key[i];
        int rank = 0;
        u64 place = place_of(cand_place[i]);
        for (int o = 0; o < n; ++o) {
            const u64 k = cand_key[o];
            rank += k > key || (k == key && o != i && place_of(cand_place[o]) < place);
        }
        if (rank >= W) continue;
        const int k = (int)(place / (unsigned)a.V), v = (int)(place - (u64)k * (unsigned)a.V);
        a.totals_out[out + rank] = (float)value_of(key);
        a.parents[out + rank] = k;
        a.classes[out + rank] = v;
        if (a.done_out) a.done_out[out + rank] = kind[k] == 2 || v == a.end;
    }
    for (int i = n + tid; i < W; i += kPickThreads) {
        a.totals_out[out + i] = -__builtin_inff();
        a.parents[out + i] = -1;
        a.classes[out + i] = -1;
        if (a.done_out) a.done_out[out + i] = 1;
    }
}

// ---- states

// One of the list's tensors: rows of `segments` stretches, of each of which the first units * unit bytes follow the beams
struct BeamState {
    char* data;
    long row, segment;                     // bytes from one row, one segment to the next
    long unit, units;                      // bytes of a position, positions
    unsigned segments;
    unsigned pad;
};
struct ReorderArgs {
    const BeamState* states;
    const int* parents;                    // [sequences][beams]
    long length;                           // positions, below zero: all
    int count, sequences, beams;
};

template <int N> struct Bytes { typedef unsigned type __attribute__((ext_vector_type(N / 4))); };
template <> struct Bytes<4> { typedef unsigned type; };
template <> struct Bytes<2> { typedef unsigned short type; };
template <> struct Bytes<1> { typedef unsigned char type; };
template <int N> struct __attribute__((packed)) AnyBytes { typename Bytes<N>::type v; };   // at any address
typedef __attribute__((address_space(1))) char global_char;        // (an address out of a table is not known to be global memory's)

// Every thread has 16 bytes (what is left of them at a segment's end) of all of a sequence's rows: it reads what its parents hold before it writes, so the
// rows change places where they lie, and a row that stays is not touched.  M: beams at most.
template <int M>
__global__ __launch_bounds__(256) void beam_reorder_kernel(ReorderArgs a)
{
    const BeamState s = a.states[blockIdx.z];
    const long bytes = (a.length >= 0 && a.length < s.units ? a.length : s.units) * s.unit;
    const unsigned along = (unsigned)((bytes + 15) / 16);
    const unsigned all = along * s.segments;             // (below 2^32: looked at when the list was made)
    if (blockIdx.x * 256u >= all) return;
    for (int q = blockIdx.y; q < a.sequences; q += gridDim.y) {
        const int* const parents = a.parents + (long)q * a.beams;
        global_char* const first = (global_char*)s.data + (long)q * a.beams * s.row;
        const int lane = threadIdx.x & 63, parent = lane < a.beams ? parents[lane] : lane;
        const int source = parent < 0 || parent >= a.beams ? lane : parent;      // (nobody's: the row stays)
        int from[M];
#pragma unroll
        for (int j = 0; j < M; ++j) from[j] = __builtin_amdgcn_readlane(source, j);
        for (unsigned i = blockIdx.x * 256u + threadIdx.x; i < all; i += gridDim.x * 256u) {
            const unsigned g = i / along, c = i - g * along;
            global_char* const at = first + g * s.segment + 16 * (long)c;
            const long left = bytes - 16 * (long)c;
            auto move = [&](auto size, global_char* p) {
                using B = __attribute__((address_space(1))) AnyBytes<decltype(size)::value>;
                typename Bytes<decltype(size)::value>::type v[M];
#pragma unroll
                for (int j = 0; j < M; ++j)
                    if (from[j] != j) v[j] = ((const B*)(p + from[j] * s.row))->v;
#pragma unroll
                for (int j = 0; j < M; ++j)
                    if (from[j] != j) ((B*)(p + j * s.row))->v = v[j];
            };
            if (left >= 16) {
                move(std::integral_constant<int, 16>{}, at);
            } else {
                global_char* p = at;
                if (left & 8) { move(std::integral_constant<int, 8>{}, p); p += 8; }
                if (left & 4) { move(std::integral_constant<int, 4>{}, p); p += 4; }
                if (left & 2) { move(std::integral_constant<int, 2>{}, p); p += 2; }
                if (left & 1) move(std::integral_constant<int, 1>{}, p);
            }
        }
    }
}

}  // namespace mpcnn
