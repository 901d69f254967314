// Beam search over many classes: which continuations go on (beam.hip), and the states that follow them.
//
//   s[k][v] = score + bias (fp32; a class whose bias is minus infinity is off),  lse[k] = log sum over v of exp s[k][v],
//   value(k, v) = total[k] + (s[k][v] - lse[k]) in 64 bits;  the `width` largest of a sequence's beams x classes, ties to the lowest beam, then class.
// A finished beam offers one candidate, the class that ends a sequence, at its total; a dead one (total minus infinity) none.
//
// Two launches.  The first goes through the scores once and is bound by memory: a wave takes steps of 1024 classes and leaves the largest score of each chunk of 256; a
// workgroup leaves its classes' largest and sum of exponentials.  The second, a workgroup per sequence, joins the sums and reads again only what can matter: the chunks whose
// largest are among the `width` best of all.  (Let an element of another chunk be among the best: `width` chunks have a largest that is better, and so is
// not below it, and these are as many elements that come before it.)  Order is by (value, then place), which no two candidates share, so the
// result does not depend on timing.  lse is a sum of fp32 exponentials, in fp32 over a workgroup's classes (a tile's), these joined in 64 bits: within one beam values are never against the scores' order.
//
// 64 sequences x 8 beams x 50021 bf16 with biases: the pass 14 us (3.7 TB/s; bound by the vector instructions: some 14 issue slots a class), the pick 9 (behind a class layer, 1 sequence x 4 beams x 32000: 8.5), a chain of
// trips to memory and LDS; chunks of 1024 instead of 256 and the best one after the other by the wave: 19 and 20 us, and 85 for 12 x 6 beams x 1573 with 16 wanted (15).
// From rows of features the first launch is the class layer's, which leaves its tiles' largest and sums beside the scores (a launch that read the scores again: 64 x 8 beams x 50021 from 4096 bf16 359 us a call,
// now 259; 128 x 4 x 50000 from 1024 200, now 86; 1 x 4 x 32000 from 1024 25.8, now 24.6).
// States: 16 x 8 beams, 16 tensors of [8][1000 of 1024][128] bf16: 1.20 ms, 5.2 TB/s.
#pragma once
#include <type_traits>

#include "any_address.hpp"
#include "lanes.hpp"

namespace mpcnn {

constexpr int kStep = 1024, kChunk = 256;  // classes
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
    int V, chunks, steps, parts, part_steps;   // chunks and steps of a row, workgroups of a row (BeamColumn: tiles), steps of a workgroup
    float2* stats;                         // [rows][stat_pitch]
    long stat_pitch;
    float* tops;                           // [rows][chunks]
    float* totals_out;
    int *parents, *classes;
    unsigned char* done_out;
};

// A row's steps: 16 lanes side by side have a chunk, a lane E numbers (16 bytes) of each J stretches of it.  The classes' shares do not depend on where the row lies, so rows that hold the same have
// the same sums (and beams that are alike are equals).
template <typename T>
struct BeamRow {
    static constexpr int E = 16 / sizeof(T), J = kStep / (64 * E);
    using Block = std::conditional_t<sizeof(T) == 2, Odd8, Raw<float, 4>>;
    const T* from;
    int V;
    bool odd;                              // begins between two words (bf16)
    const float* bias;
    __device__ BeamRow(const BeamArgs& a, long row) : from((const T*)a.scores + row * a.pitch), V(a.V), odd((uintptr_t)from & 2), bias(a.bias) {}
    __device__ static int number(int j) { return kChunk * (int)(threadIdx.x >> 4 & 3) + E * ((int)(threadIdx.x & 15) + 16 * j); }
    __device__ void fetch(int step, Block (&u)[J]) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = kStep * step + number(j);
            if (at >= V) continue;
            if constexpr (sizeof(T) == 4) u[j] = raw_of<4>(from, at, V);
            else if (at + 8 > V) u[j] = odd8_of(from, at, V);
            else if (odd) u[j] = odd8(from + at);
            else u[j].a = *reinterpret_cast<const Odd8::u4_any*>(from + at);
        }
    }
    // scores with the bias; minus infinity beyond the row and for classes that are off, whatever is there.  SIMPLE: of a whole step, in which a class that is off
    // may be NaN if its score is not finite
    template <bool SIMPLE = false>
    __device__ void scores(int step, const Block (&u)[J], float (&s)[J][E]) const
    {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int at = kStep * step + number(j);
            float b[E];
            if (bias && (SIMPLE || at + E <= V)) {
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const f4_any w = *reinterpret_cast<const f4_any*>(bias + at + e);
#pragma unroll
                    for (int z = 0; z < 4; ++z) b[e + z] = w[z];
                }
            } else if constexpr (SIMPLE) {
#pragma unroll
                for (int e = 0; e < E; ++e) b[e] = 0.f;
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
            for (int e = 0; e < E; ++e) s[j][e] = SIMPLE || (at + e < V && b[e] != -__builtin_inff()) ? s[j][e] + b[e] : -__builtin_inff();
        }
    }
    // one of them
    __device__ float one(int at) const
    {
        const float b = bias && at < V ? bias[at] : 0.f;
        return at < V && b != -__builtin_inff() ? load1(from + at) + b : -__builtin_inff();
    }
    static constexpr int kParts = 1;       // so many a lane at once
    // the first launch's: of a part of a row's classes, and the largest of chunk i of the chunks of all of a sequence's beams
    __device__ static float2 stat(const BeamArgs& a, long row, int part) { return a.stats[row * a.stat_pitch + part]; }
    __device__ static float top(const BeamArgs& a, long row0, int i) { return a.tops[row0 * a.chunks + i]; }
};

// exp(x - top) for x <= top; 0 for minus infinity
__device__ __forceinline__ float exp_below(float x, float top) { return __builtin_amdgcn_exp2f((x - top) * 1.4426950408889634f); }

// Scores that lie [class][row], fp32, as a class layer leaves them, with their bias, and what it leaves of its tiles of classes, PER of which are a chunk
template <int PER>
struct BeamColumn {
    static constexpr int kParts = PER > 4 ? 16 : 8;      // (1 x 4 x 32000, 1000 tiles, joined in 32 bits: 24.1 us a call, with 8 24.9)
    const float* from;
    long pitch;
    int V;
    __device__ BeamColumn(const BeamArgs& a, long row) : from((const float*)a.scores + row), pitch(a.pitch), V(a.V) {}
    __device__ float one(int at) const { return at < V ? from[at * pitch] : -__builtin_inff(); }
    __device__ static float2 stat(const BeamArgs& a, long row, int part) { return a.stats[row * a.stat_pitch + part]; }
    __device__ static float top(const BeamArgs& a, long row0, int i)
    {
        const int k = i / a.chunks, first = PER * (i - k * a.chunks);
        float t[PER];
#pragma unroll
        for (int q = 0; q < PER; ++q) t[q] = stat(a, row0 + k, first + q < a.parts ? first + q : a.parts - 1).x;      // (the last chunk's, again)
#pragma unroll
        for (int q = 1; q < PER; ++q) t[0] = fmaxf(t[0], t[q]);
        return t[0];
    }
};

// A part's sum, of exponentials below the largest of all parts, in 64 bits
__device__ __forceinline__ double share(const float2& s, float top) { return s.x > -__builtin_inff() || s.y != 0.f ? (double)s.y * exp((double)s.x - (double)top) : 0.0; }
// Of some parts, with half the instructions: exponentials to 2^-38 of themselves, 1 for the largest.  2^f on [-1/2, 1/2] is 1 + f q(f), q through (2^f - 1) / f at Chebyshev's eight points.
template <int N>
__device__ __forceinline__ double shares(const float2 (&s)[N], float top)
{
    constexpr double q[8] = {0.6931471805568324, 0.24022650695888503, 0.055504109063258665, 0.00961812913523614, 0.0013333478473685416, 0.00015403475186530786, 1.5303700711365693e-05, 1.325080551750225e-06};
    double f[N], p[N], sum = 0.0;
    int n[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {                        // (no part's largest, or no number: 2^-1000 times what the sum is)
        const double t = fmax(((double)s[k].x - (double)top) * 1.4426950408889634, -1000.0), whole = rint(t);
        n[k] = (int)whole;
        f[k] = t - whole;
        p[k] = q[7];
    }
#pragma unroll
    for (int i = 6; i >= 0; --i)
#pragma unroll
        for (int k = 0; k < N; ++k) p[k] = fma(p[k], f[k], q[i]);
#pragma unroll
    for (int k = 0; k < N; ++k) sum += (double)s[k].y * ldexp(fma(p[k], f[k], 1.0), n[k]);
    return sum;
}

__device__ __forceinline__ bool beam_goes_on(const BeamArgs& a, long row)
{
    return fabsf(a.totals[row]) < __builtin_inff() && !(a.done && a.done[row]);     // (a NaN does not)
}

// Largest and sum of exponentials of two lots of classes together
__device__ __forceinline__ float2 joined(const float2& p, const float2& q)
{
    const float now = fmaxf(p.x, q.x), base = now == -__builtin_inff() ? 0.f : now;
    return float2{now, p.y * exp_below(p.x, base) + q.y * exp_below(q.x, base)};
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
    const int end = (part + 1) * a.part_steps < a.steps ? (part + 1) * a.part_steps : a.steps;
    int c = part * a.part_steps + wave;
    typename Row::Block u[Row::J];
    if (c < end) r.fetch(c, u);
    float top = -__builtin_inff(), sum = 0.f;
    for (; c < end; c += 4) {
        float s[Row::J][Row::E], now, more;
        auto add = [&] {
            float most = s[0][0];
#pragma unroll
            for (int j = 0; j < Row::J; ++j)
#pragma unroll
                for (int e = 0; e < Row::E; ++e) most = fmaxf(most, s[j][e]);
            most = largest16(most);
            const int chunk = kStep / kChunk * c + (lane >> 4);
            if ((lane & 15) == 0 && chunk < a.chunks) a.tops[row * a.chunks + chunk] = most;
            now = fmaxf(top, largest_of16s(most));
            const float base = now == -__builtin_inff() ? 0.f : now;
            more = 0.f;
#pragma unroll
            for (int j = 0; j < Row::J; ++j)
#pragma unroll
                for (int e = 0; e < Row::E; ++e) more += exp_below(s[j][e], base);
        };
        const bool whole = kStep * (c + 1) <= a.V;
        if (whole) {
            r.template scores<true>(c, u, s);
            add();
        }
        if (!whole || (a.bias && __ballot(more != more))) {   // (hardly ever)
            r.scores(c, u, s);
            add();
        }
        if (c + 4 < end) r.fetch(c + 4, u);
        sum = sum * exp_below(top, now == -__builtin_inff() ? 0.f : now) + more;
        top = now;
    }
    sum = sum64(sum);
    if (lane == 0) red[wave] = float2{top, sum};
    __syncthreads();
    if (threadIdx.x == 0) {
        float2 all = red[0];
#pragma unroll
        for (int w = 1; w < 4; ++w) all = joined(all, red[w]);
        a.stats[row * a.stat_pitch + part] = all;
    }
}

// ---- the second launch

typedef unsigned long long u64;
// Values in an order of whole numbers; 0: no candidate
__device__ __forceinline__ u64 key_of(double v)
{
    if (!(v > -__builtin_inf())) return 0;
    const u64 b = __builtin_bit_cast(u64, v + 0.0);      // (minus zero is zero's equal)
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double value_of(u64 key) { return __builtin_bit_cast(double, key >> 63 ? key ^ 1ull << 63 : ~key); }

// A chunk or a candidate and its place among those of the same value: the lower one is better
struct Offer { u64 key; unsigned place; };
__device__ __forceinline__ bool better(const Offer& a, const Offer& b) { return a.key > b.key || (a.key == b.key && a.place < b.place); }
// The better one of this lane's and of the one that CTRL names
template <int CTRL>
__device__ __forceinline__ Offer better_moved(const Offer& m)
{
    auto moved = [](unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false); };
    const Offer o{(u64)moved((unsigned)(m.key >> 32)) << 32 | moved((unsigned)m.key), moved(m.place)};
    return better(o, m) ? o : m;
}
// Over `lanes` (2, 4 or 8, uniform) side by side, in all of them
__device__ __forceinline__ Offer best_beside(Offer m, int lanes)
{
    m = better_moved<0xb1>(m);                       // quad_perm:[1,0,3,2]
    if (lanes > 2) m = better_moved<0x4e>(m);        // quad_perm:[2,3,0,1]
    return lanes > 4 ? better_moved<0x141>(m) : m;   // row_half_mirror
}
__device__ __forceinline__ int sum_beside(int v, int lanes)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true);
    if (lanes > 2) v += __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true);
    return lanes > 4 ? v + __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, true) : v;
}

// What is picked from is kept in LDS: places for kSpare offers of each wanted one (kEach of each of a group's threads, and the winners so far)
constexpr int kEach = 8, kSpare = 8 * kEach + 1;
constexpr size_t pick_bytes(int width) { return (size_t)width * (width > kSpare ? width : kSpare) * 12; }

template <typename Row>
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(BeamArgs a)
{
    constexpr int kGroups = kPickThreads / 2;
    extern __shared__ __attribute__((aligned(16))) char lds_raw[];
    __shared__ double lse[kMaxBeams];
    __shared__ float total[kMaxBeams];
    __shared__ int kind[kMaxBeams];                      // 0: offers nothing, 1: goes on, 2: finished
    __shared__ u64 group_key[kGroups];
    __shared__ unsigned group_place[kGroups];
    __shared__ u64 chosen_key[kMaxBeams];
    __shared__ unsigned chosen_place[kMaxBeams], number_of[kMaxBeams], numbered[kMaxBeams];
    __shared__ u64 least_key;
    __shared__ unsigned least_place, count;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // threads of a group, so that there are four groups for every wanted one
    const int beside = a.width <= kPickThreads / 32 ? 8 : a.width <= kPickThreads / 16 ? 4 : 2, of_group = tid / beside;
    static_assert(kMaxBeams <= kPickThreads / 8, "groups of two do");
    const int W = a.width, K = a.beams, all = K * a.chunks;            // (chunks of all beams: below 2^30)
    const int room = W * (W > kSpare ? W : kSpare);
    u64* const cand_key = reinterpret_cast<u64*>(lds_raw);             // [room]
    unsigned* const cand_place = reinterpret_cast<unsigned*>(lds_raw + sizeof(u64) * room);
    const long row0 = (long)blockIdx.x * K;

    float tops[kEach];
    auto fetch = [&](int base) {
#pragma unroll
        for (int r = 0; r < kEach; ++r) {
            const int i = base + kPickThreads * r + tid;
            tops[r] = i < all ? Row::top(a, row0, i) : 0.f;     // (of a beam that does not go on: whatever is there)
        }
    };
    fetch(0);

    // ---- the beams' sums
    for (int k = wave; k < K; k += kPickWaves) {
        const long row = row0 + k;
        const float t = a.totals[row];
        const bool over = a.done && a.done[row];
        float2 mine[Row::kParts];                        // (used if it goes on)
        constexpr int kBeside = 64 * Row::kParts;
        auto part = [&](int p) { return p < a.parts ? Row::stat(a, row, p) : float2{-__builtin_inff(), 0.f}; };
#pragma unroll
        for (int q = 0; q < Row::kParts; ++q) mine[q] = part(64 * q + lane);
        int is = fabsf(t) < __builtin_inff() ? (over ? 2 : 1) : 0;
        double l = 0.0;
        if (is == 1) {
            float top = mine[0].x;
#pragma unroll
            for (int q = 1; q < Row::kParts; ++q) top = fmaxf(top, mine[q].x);
#pragma unroll 4
            for (int p = kBeside + lane; p < a.parts; p += 64) top = fmaxf(top, Row::stat(a, row, p).x);
            top = largest64(top);
            double sum = 0.0;
            if constexpr (Row::kParts == 1) {
                sum = share(mine[0], top);
#pragma unroll 4
                for (int p = kBeside + lane; p < a.parts; p += 64) sum += share(Row::stat(a, row, p), top);
            } else {                                     // (there are many)
                float2 some[4];
#pragma unroll 1
                for (int q = 0; q < Row::kParts; q += 4) {             // (one copy of it, instructions come from memory, too: 1 x 4 x 32000 from 1024 24.6 us a call, four copies 25.4)
#pragma unroll
                    for (int z = 0; z < 4; ++z) some[z] = mine[z];
#pragma unroll
                    for (int z = 0; z + 4 < Row::kParts; ++z) mine[z] = mine[z + 4];
                    sum += shares(some, top);
                }
                for (int p = kBeside + lane; p < a.parts; p += 4 * 64) {
#pragma unroll
                    for (int z = 0; z < 4; ++z) some[z] = part(p + 64 * z);
                    sum += shares(some, top);
                }
            }
#pragma unroll
            for (int i = 1; i < 64; i *= 2) sum += __shfl_xor(sum, i, 64);
            l = (double)top + log(sum);
            if (!(l > -__builtin_inf() && l < __builtin_inf())) is = 0;        // nothing is on, or a score is not finite
        }
        if (lane == 0) { lse[k] = l; total[k] = t; kind[k] = is; }
    }
    if (tid < W) { chosen_key[tid] = 0; chosen_place[tid] = 0xffffffffu; }
    __syncthreads();

    auto rank_of = [&](const Offer& mine, int n) {           // how many of the first n candidates come before
        int rank = 0;
#pragma unroll 4
        for (int o = 0; o < n; ++o) rank += better(Offer{cand_key[o], cand_place[o]}, mine);
        return rank;
    };
    // The best W of the first `n` candidates into chosen, best first, by how many come before each
    auto choose = [&](int n) {
        for (int i = tid; i < n; i += kPickThreads) {
            const Offer mine{cand_key[i], cand_place[i]};
            const int rank = rank_of(mine, n);
            if (rank < W) { chosen_key[rank] = mine.key; chosen_place[rank] = mine.place; }
        }
    };
    auto offer = [&](u64 key, unsigned place) {
        const unsigned i = atomicAdd(&count, 1u);
        cand_key[i] = key;
        cand_place[i] = place;
    };

    // ---- the best chunks, kEach of a thread at a time: no better ones than those that are not worse than the W-th best of the groups' best can be among the best W
    for (int base = 0; base < all; base += kPickThreads * kEach) {
        Offer mine[kEach], best{0, 0xffffffffu};
#pragma unroll
        for (int r = 0; r < kEach; ++r) {
            const int i = base + kPickThreads * r + tid;
            mine[r] = Offer{0, (unsigned)i};
            if (i >= all) continue;
            const int k = i / a.chunks;
            if (kind[k] == 1) mine[r].key = key_of((double)total[k] + ((double)tops[r] - lse[k]));
            else if (kind[k] == 2 && i == k * a.chunks) mine[r].key = key_of((double)total[k]);        // (its one candidate)
            if (better(mine[r], best)) best = mine[r];
        }
        if (base + kPickThreads * kEach < all) fetch(base + kPickThreads * kEach);
        best = best_beside(best, beside);
        if (tid % beside == 0) { group_key[of_group] = best.key; group_place[of_group] = best.place; }
        if (tid == 0) { least_key = 0; least_place = 0xffffffffu; count = 0; }
        __syncthreads();
        {   // a group's threads: how many groups' best come before its
            int rank = 0;
            for (int g = tid % beside; g < kPickThreads / beside; g += beside) rank += better(Offer{group_key[g], group_place[g]}, best);
            rank = sum_beside(rank, beside);
            if (rank == W - 1 && tid % beside == 0 && best.key) { least_key = best.key; least_place = best.place; }     // (groups without a chunk are alike)
        }
        __syncthreads();
        const Offer least{least_key, least_place};
#pragma unroll
        for (int r = 0; r < kEach; ++r)
            if (mine[r].key && !better(least, mine[r])) offer(mine[r].key, mine[r].place);
        if (base && tid < W && chosen_key[tid]) offer(chosen_key[tid], chosen_place[tid]);
        __syncthreads();
        const int n = (int)count;
        if (base) {                                      // (the winners so far are candidates now)
            if (tid < W) { chosen_key[tid] = 0; chosen_place[tid] = 0xffffffffu; }
            __syncthreads();
        }
        choose(n);
        __syncthreads();
    }
    // (candidates' places have to be in the order of their beams and classes: the chosen chunks are numbered by their places)
    if (tid < W) {
        const unsigned mine = chosen_place[tid];
        int n = 0;
        for (int o = 0; o < W; ++o) n += chosen_place[o] < mine;
        number_of[tid] = (unsigned)n << 8;
        if (chosen_key[tid]) numbered[n] = mine;
    }
    if (tid == 0) count = 0;
    __syncthreads();

    // ---- their numbers that are not below the last chosen chunk's largest (of a chunk with many: the best)
    constexpr int E = kChunk / 64;
    const u64 least = chosen_key[W - 1];
    float next[E];
    auto look = [&](int w) {
        if (w >= W || !chosen_key[w]) return;
        const int k = (int)(chosen_place[w] / (unsigned)a.chunks), c = (int)chosen_place[w] - k * a.chunks;
        if (kind[k] == 2) return;
        const Row r(a, row0 + k);
#pragma unroll
        for (int e = 0; e < E; ++e) next[e] = r.one(kChunk * c + E * lane + e);
    };
    look(wave);
    for (int w = wave; w < W; w += kPickWaves) {
        if (!chosen_key[w]) continue;
        const int k = (int)(chosen_place[w] / (unsigned)a.chunks);
        if (kind[k] == 2) {
            if (lane == 0) offer(chosen_key[w], number_of[w]);
            look(w + kPickWaves);
            continue;
        }
        float s[E];
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] = next[e];
        look(w + kPickWaves);
        // a score below `lo` has a value below the least (a millionth is more than the roundings)
        const double t = (double)total[k], need = least ? value_of(least) - t + lse[k] : -__builtin_inf();
        const float lo = (float)(need - 1e-6 * (fabs(need) + fabs(t) + fabs(lse[k])));
        u64 key[E];
        int n = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            key[e] = 0;
            if (s[e] >= lo && s[e] > -__builtin_inff()) {
                const u64 v = key_of(t + ((double)s[e] - lse[k]));
                if (v >= least) key[e] = v;
            }
            n += __builtin_popcountll(__ballot(key[e] != 0));
        }
        const unsigned of = number_of[w];
        static_assert(kChunk == 256, "a number's bits");
        if (n > (W > kSpare ? W : kSpare)) {             // more than there is room for: those that are not worse than the W-th best of the lanes' best
            Offer best{0, 0xffffffffu};
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (key[e] > best.key) best = Offer{key[e], (unsigned)(E * lane + e)};
            int rank = 0;
#pragma unroll
            for (int l = 0; l < 64; ++l) {
                const Offer o{(u64)(unsigned)__builtin_amdgcn_readlane((int)(best.key >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)best.key, l),
                              (unsigned)__builtin_amdgcn_readlane((int)best.place, l)};
                rank += better(o, best);
            }
            const u64 last = __ballot(rank == W - 1 && best.key != 0);
            if (last) {
                const int l = __builtin_ctzll(last);
                const u64 bound = (u64)(unsigned)__builtin_amdgcn_readlane((int)(best.key >> 32), l) << 32 | (unsigned)__builtin_amdgcn_readlane((int)best.key, l);
                n = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    key[e] = key[e] >= bound ? key[e] : 0;
                    n += __builtin_popcountll(__ballot(key[e] != 0));
                }
            }
        }
        if (n <= (W > kSpare ? W : kSpare)) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (key[e]) offer(key[e], of | (unsigned)(E * lane + e));
            continue;
        }
        for (int q = 0; q < W; ++q) {                    // (more than can be: the best of them, one after the other)
            Offer best{0, 0xffffffffu};
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const Offer o{key[e], (unsigned)(E * lane + e)};
                if (better(o, best)) best = o;
            }
            best = best_beside(best, 8);
            best = better_moved<0x128>(best);            // row_ror:8
#pragma unroll
            for (int i = 16; i < 64; i *= 2) {
                const Offer o{__shfl_xor(best.key, i, 64), __shfl_xor(best.place, i, 64)};
                if (better(o, best)) best = o;
            }
            if (!best.key) break;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (best.place == (unsigned)(E * lane + e)) key[e] = 0;
            if (lane == 0) offer(best.key, of | best.place);
        }
    }
    __syncthreads();

    // ---- the best of these
    const int n = (int)count;
    const long out = (long)blockIdx.x * W;
    for (int i = tid; i < n; i += kPickThreads) {
        const Offer mine{cand_key[i], cand_place[i]};
        const int rank = rank_of(mine, n);
        if (rank >= W) continue;
        const unsigned chunk = numbered[mine.place >> 8];
        const int k = (int)(chunk / (unsigned)a.chunks), c = (int)chunk - k * a.chunks;
        const int v = kind[k] == 2 ? a.end : kChunk * c + (int)(mine.place & (kChunk - 1));
        a.totals_out[out + rank] = (float)value_of(mine.key);
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
    int sequences, beams;
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
