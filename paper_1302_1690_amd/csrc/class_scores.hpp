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
// The scores with their bias, fp32 [classes][*row], in the workspace
mpcnn_status class_scores(const ClassScores& c, char* ws, float** scores, int64_t* row, hipStream_t st);

}  // namespace mpcnn
