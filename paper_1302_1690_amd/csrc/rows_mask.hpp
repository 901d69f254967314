// Which rows of features count, and the derivative of their loss (class_rows.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace mpcnn {

// Rows that add something: a label among the classes and a weight that is not zero
struct RowMask {
    const int* labels;
    const float* weights;                  // null: 1
    int classes;
};
__device__ __forceinline__ float row_weight(const RowMask& m, int n)
{
    const int t = m.labels[n];
    if (t < 0 || t >= m.classes) return 0.f;
    return m.weights ? m.weights[n] : 1.f;
}

// exp(score - lse) - hot; nothing for rows that are not live.  exp by the hardware's exp2, whose argument's rounding is made good: x log2 e = t + r
// to twice fp32's bits, 2^(t + r) = 2^t (1 + r ln 2) for |r| below a 2^-24th of t.
constexpr float kLog2eHigh = 1.4426950408889634f, kLog2eLow = 1.925963033500212e-08f;   // log2 e in two fp32 numbers
__device__ __forceinline__ float class_delta(float score, float lse, bool live, bool hot)
{
    const float x = score == -__builtin_inff() ? -1e30f : score - lse;     // (a class that is switched off, and a row that has no other)
    const float t = x * kLog2eHigh, r = fmaf(x, kLog2eHigh, -t) + x * kLog2eLow;
    const float e = __builtin_amdgcn_exp2f(t);
    const float p = e > 0.f ? fmaf(e, r * 0.6931471805599453f, e) : e;
    return live ? (hot ? p - 1.f : p) : 0.f;
}

constexpr int kNoLabel = -1;               // in the place of the label of a row that adds nothing

}  // namespace mpcnn
