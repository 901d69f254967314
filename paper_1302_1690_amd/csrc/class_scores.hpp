// A class layer's scores on few rows of features, all of them kept (class_rows.hip), for what picks classes by them (beam.hip).
#pragma once
#include <cstdint>

#include "status.hpp"

namespace mpcnn {

struct ClassScores {
    const void *x, *w;                     // [rows][x_pitch], [classes][w_pitch]
    int64_t x_pitch, w_pitch;
    const float* bias;                     // or null
    int64_t rows, features, classes;
    int dtype;
};
size_t class_scores_bytes(const ClassScores& c);         // of the workspace; it grows with the rows.  0: bad or too large
// In the workspace: the scores with their bias, fp32 [classes][row], and the largest and the sum of exp(score - largest) of each tile of so many classes
// (32, 64, 128 or 256), [rows][stat_pitch]
struct KeptScores {
    float* scores;
    int64_t row;
    float2* stats;
    int64_t stat_pitch, tile, tiles;
};
mpcnn_status class_scores(const ClassScores& c, char* ws, KeptScores* kept, hipStream_t st);

}  // namespace mpcnn
