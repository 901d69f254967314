// Launches of the update kernels (update.hip, kernels_update.hpp), for lists of tensors and for a net's own parameters.
#pragma once
#include <hip/hip_runtime.h>

namespace mpcnn {

constexpr int kNormParts = 1024;           // most partial sums
constexpr unsigned kStretch = 8192;        // most numbers of a stretch
constexpr unsigned kStretchLeast = 512;    // one fetch of every lane
constexpr long kLoneNumbers = 16384;
constexpr int kLoneStretches = 64;

struct Stretch {
    void* grad;
    void* param;            // null where there are no parameters
    unsigned n;
    unsigned short grad_bf16, param_bf16;
};
struct UpdateArgs {
    const Stretch* table;   // null: `flat`, cut into stretches of flat_len
    Stretch flat;
    long flat_n;
    unsigned flat_len;
    int stretches, parts;
    double* partial;        // [parts]
    double* norm;           // result, or null
    double scale, bound;    // |s|, largest norm
    double rate;            // signed: rate * s
};
enum { kOnlyNorm = 0, kClip = 1, kStep = 2 };

// Whether a step can be taken with these numbers: each finite, and so the product, as an fp32 number too
bool rate_fits(double rate, double scale);
// Stretch length for so many numbers in all: enough stretches for every wave that can run, none shorter than one fetch
unsigned stretch_length(long total);
// mode: kOnlyNorm, kClip, kStep; fills in a.parts.  `total`: numbers in all.  Where tensors that are written share memory, they are updated in runs, one
// after the other, in the list's order: starts[0 .. runs] are the runs' stretches (runs = 0: no two do).
void launch_update(UpdateArgs a, int mode, long total, const int* starts, int runs, hipStream_t st);

}  // namespace mpcnn
