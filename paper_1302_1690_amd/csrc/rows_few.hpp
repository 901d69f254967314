// The launches of the class layer on few rows of features (rows_few.hip, kernels_rows_few.hpp).
#pragma once
#include "rows_mask.hpp"

namespace mpcnn {

constexpr int kFewRows = 16, kFewScoreRows = 12, kFewRound = 64;      // rows, classes of a round
constexpr int kFewThreads = 256;
// Features of a thread of rows_few_grads: what a thread keeps of every row and of its gradient fits its registers
__host__ __device__ constexpr int few_columns(int rows) { return rows <= 8 ? 8 : 4; }

struct FewArgs {
    const void *x, *w;
    long x_pitch, w_pitch;
    int N, D;
    long V, score_row;
    const float* bias;
    RowMask mask;
    float* scores;                               // [V][score_row], or null
    float2* stats;                               // [workgroups][N]
    float* label_score;
    long each;                                   // classes of a workgroup
    // gradients
    const float *lse, *weight;
    void* dw;
    float *db, *part;                            // part: [workgroups][N][D] shares of dx, or null
    int columns;                                 // threads that share a class's features: 16 .. 256, a power of two
    // sum
    int parts;
    void* dx;
    long dx_pitch;
    const double* loss_part;
    int loss_parts;
    double* loss;
};

template <typename T> void launch_rows_few_scores(const FewArgs& a, unsigned groups, hipStream_t st); // a.N = 1 .. kFewScoreRows
template <typename T> void launch_rows_few_grads(const FewArgs& a, dim3 grid, hipStream_t st);        // a.N = 1 .. kFewRows
template <typename T> void launch_rows_few_sum(const FewArgs& a, unsigned groups, hipStream_t st);

}  // namespace mpcnn
