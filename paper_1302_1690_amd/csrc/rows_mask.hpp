// Which rows of features count (class_rows.hip).
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

constexpr int kNoLabel = -1;               // in the place of the label of a row that adds nothing

}  // namespace mpcnn
