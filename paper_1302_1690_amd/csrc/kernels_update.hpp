// The update step on lists of tensors (Results, "Membrane Segmentation": weights updated after every image): the 2-norm over all
// gradients together, gradients scaled down to a bound on it, and the gradient step with the same factor,
//     norm = |s| sqrt(sum g^2),   c = min(1, bound / norm),   g <- c g   or   theta <- theta - rate s c g.
//
// Two launches: partial sums of squares, one per workgroup; then every workgroup adds the partial sums (all in the same fixed order, so
// all hold the same norm and no grid-wide wait is needed) and updates its share.  Lists that one workgroup sees through (kLoneNumbers)
// take one launch.  Squares and sums are fp64: a square of an fp32 number is exact in it, and none overflows.  The work is dealt to
// waves in stretches of at most kStretch numbers of one tensor, dealt out in the list's order.  A tensor may start at any element:
// lanes fetch 8 numbers as one or two 128-bit words at whatever address they have.
//
// The factor c, or rate s c, is rounded to fp32 once.  Below fp32's normal numbers it would lose bits there, or all of them (gradients of 1e38 clipped to a norm of
// 1): then it is taken as `lift` = 2^-126, by which gradients are multiplied first, exactly where it matters, and what is left of it.
//
// A norm that is not finite (an infinity or NaN among the gradients) changes nothing: gradients and parameters stay as they were.
//
// Bound by the passes over memory: one for the norm, two more for clipping (none where the norm is within the bound: the gradients
// are what they were), three more for a step.  5e8 numbers of both types in 300 tensors: norm 237 us, 5.6 TB/s.  4e8 fp32 numbers in 300 tensors: step
// 1205 us, 5.3 TB/s over four passes.  80e6 bf16 numbers in 150 tensors: clipping 141 us with the copy that brings the gradients.  3e6 in 1000 tensors:
// 11 us, two launches.  The update goes through the list from its end on: what the norm's pass read last is in the last-level cache (steps on
// 1e8 fp32 numbers 327 -> 307 us, on 4e8 1230 -> 1205, on 1.5e8 bf16 250 -> 237).
#pragma once
#include "any_address.hpp"
#include "update.hpp"

namespace mpcnn {

__device__ __forceinline__ Stretch stretch_at(const UpdateArgs& a, int s)
{
    if (a.table) return a.table[s];
    Stretch t = a.flat;
    const long at = (long)s * a.flat_len, left = a.flat_n - at;
    t.grad = (char*)t.grad + at * (t.grad_bf16 ? 2 : 4);
    if (t.param) t.param = (char*)t.param + at * (t.param_bf16 ? 2 : 4);
    t.n = left < a.flat_len ? (unsigned)left : a.flat_len;
    return t;
}

template <typename G>
__device__ __forceinline__ double squares(const G* g, unsigned n, unsigned lane)
{
    double s0 = 0.0, s1 = 0.0;
    auto add = [&](v8f v) {
#pragma unroll
        for (int z = 0; z < 8; z += 2) {
            s0 = fma((double)v[z], (double)v[z], s0);
            s1 = fma((double)v[z + 1], (double)v[z + 1], s1);
        }
    };
    unsigned i = 8 * lane;
    for (; i + 3 * 512 + 8 <= n; i += 4 * 512) {       // four fetches in flight
        v8f v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = load8(g + i + 512 * q);
#pragma unroll
        for (int q = 0; q < 4; ++q) add(v[q]);
    }
    for (; i + 8 <= n; i += 512) add(load8(g + i));
    const unsigned t = (n & ~7u) + lane;
    if (t < n) {
        const double x = (double)load1(g + t);
        s0 = fma(x, x, s0);
    }
    return s0 + s1;
}

template <typename G>
__device__ __forceinline__ void scale_down(G* g, unsigned n, unsigned lane, float c, float lift)
{
    unsigned i = 8 * lane;
    for (; i + 3 * 512 + 8 <= n; i += 4 * 512) {
        v8f v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = load8(g + i + 512 * q);
#pragma unroll
        for (int q = 0; q < 4; ++q) store8(g + i + 512 * q, v[q] * lift * c);
    }
    for (; i + 8 <= n; i += 512) store8(g + i, load8(g + i) * lift * c);
    const unsigned t = (n & ~7u) + lane;
    if (t < n) store1(g + t, load1(g + t) * lift * c);
}

__device__ __forceinline__ v8f moved(v8f p, v8f g, float f, float lift)
{
#pragma unroll
    for (int z = 0; z < 8; ++z) p[z] = fmaf(-f, g[z] * lift, p[z]);
    return p;
}
template <typename G, typename P>
__device__ __forceinline__ void step_down(const G* g, P* p, unsigned n, unsigned lane, float f, float lift)
{
    unsigned i = 8 * lane;
    for (; i + 512 + 8 <= n; i += 2 * 512) {
        const v8f g0 = load8(g + i), g1 = load8(g + i + 512), p0 = load8(p + i), p1 = load8(p + i + 512);
        store8(p + i, moved(p0, g0, f, lift));
        store8(p + i + 512, moved(p1, g1, f, lift));
    }
    for (; i + 8 <= n; i += 512) store8(p + i, moved(load8(p + i), load8(g + i), f, lift));
    const unsigned t = (n & ~7u) + lane;
    if (t < n) store1(p + t, fmaf(-f, load1(g + t) * lift, load1(p + t)));
}

// Sum over the workgroup's threads in a fixed order; the result in every thread
template <int WAVES>
__device__ __forceinline__ double group_sum(double v, double* red)
{
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) v += __shfl_down(v, w, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += red[w];
    return s;
}

// Squares of the stretches first, first + by, ...
__device__ __forceinline__ double squares_of(const UpdateArgs& a, int first, int by, unsigned lane)
{
    double s = 0.0;
    for (int i = first; i < a.stretches; i += by) {
        const Stretch t = stretch_at(a, i);
        s += t.grad_bf16 ? squares((const bf16*)t.grad, t.n, lane) : squares((const float*)t.grad, t.n, lane);
    }
    return s;
}

__global__ __launch_bounds__(256) void norm_parts_kernel(UpdateArgs a)
{
    __shared__ double red[4];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const double s = group_sum<4>(squares_of(a, (int)blockIdx.x * 4 + wave, (int)gridDim.x * 4, threadIdx.x & 63), red);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = s;
}

template <int MODE, bool LONE>
__global__ __launch_bounds__(LONE ? 1024 : 256) void update_kernel(UpdateArgs a)
{
    constexpr int WAVES = LONE ? 16 : 4;
    __shared__ double red[WAVES];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned lane = threadIdx.x & 63;
    double s = 0.0;
    if constexpr (LONE) {
        s = squares_of(a, wave, WAVES, lane);
    } else {
        double v[kNormParts / 256];
#pragma unroll
        for (int q = 0; q < kNormParts / 256; ++q) {
            const int at = 256 * q + (int)threadIdx.x;
            v[q] = at < a.parts ? a.partial[at] : 0.0;
        }
#pragma unroll
        for (int q = 0; q < kNormParts / 256; ++q) s += v[q];
    }
    const double norm = a.scale * sqrt(group_sum<WAVES>(s, red));
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm) *a.norm = norm;
    if constexpr (MODE == kOnlyNorm) return;
    if (!(norm < __builtin_inf())) return;                   // (NaN too)
    const double c = norm > a.bound ? a.bound / norm : 1.0;
    if (MODE == kClip && c == 1.0) return;
    const double factor = MODE == kClip ? c : c * a.rate;
    const bool low = fabs(factor) < 0x1p-126;
    const float f = (float)(low ? factor * 0x1p126 : factor), lift = low ? 0x1p-126f : 1.f;   // one rounding; the product with a gradient is the next
    const int first = (int)blockIdx.x * WAVES + wave, by = (int)gridDim.x * WAVES;
    for (int i = first; i < a.stretches; i += by) {
        const Stretch t = stretch_at(a, LONE ? i : a.stretches - 1 - i);   // (from the end on)
        if constexpr (MODE == kClip) {
            if (t.grad_bf16) scale_down((bf16*)t.grad, t.n, lane, f, lift);
            else scale_down((float*)t.grad, t.n, lane, f, lift);
        } else if (t.grad_bf16) {
            if (t.param_bf16) step_down((const bf16*)t.grad, (bf16*)t.param, t.n, lane, f, lift);
            else step_down((const bf16*)t.grad, (float*)t.param, t.n, lane, f, lift);
        } else {
            if (t.param_bf16) step_down((const float*)t.grad, (bf16*)t.param, t.n, lane, f, lift);
            else step_down((const float*)t.grad, (float*)t.param, t.n, lane, f, lift);
        }
    }
}

}  // namespace mpcnn
