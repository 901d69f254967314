// Beam search over many classes: the continuations that go on, and the beams' states (include/mpcnn.h, mpcnn_beam_select and what follows): checks and launches.
#include <algorithm>
#include <cstdint>
#include <memory>
#include <new>
#include <numeric>
#include <vector>

#include "class_scores.hpp"
#include "kernels_beam.hpp"
#include "spans.hpp"
#include "status.hpp"

using mpcnn::fail;
using mpcnn::meet;
using mpcnn::Span;

struct mpcnn_beam_states {
    int device = -1;
    int count = 0, sequences = 0, beams = 0;
    std::vector<mpcnn::BeamState> states;
    std::vector<Span> held;                // the tensors' memory
    mpcnn::BeamState* d_states = nullptr;
};

namespace {

constexpr int64_t kMaxRows = 1 << 20, kMaxClasses = 0x7fffffff - 1024, kMostPitch = (int64_t)1 << 40;
constexpr int64_t kMostScores = (int64_t)1 << 34;      // of a class layer, kept (64 GB)
constexpr int kCUs = 256;

struct Plan { int64_t rows, chunks, steps, parts, part_steps; size_t stats, tops, total; };

// columns: the scores are a class layer's, [class][row], which has left what the first launch would
bool make_plan(int64_t sequences, int64_t beams, int64_t classes, Plan* p, bool columns = false)
{
    if (sequences < 0 || beams < 1 || beams > mpcnn::kMaxBeams || sequences > kMaxRows / beams || classes < 1 || classes > kMaxClasses) return false;
    *p = Plan{};
    p->rows = sequences * beams;
    p->chunks = (classes + mpcnn::kChunk - 1) / mpcnn::kChunk;
    if (columns) return p->rows * classes <= kMostScores;
    p->steps = (classes + mpcnn::kStep - 1) / mpcnn::kStep;
    // eight workgroups a compute unit, each wave of which has a step at least
    const int64_t wanted = std::max<int64_t>(1, 8 * kCUs / std::max<int64_t>(1, p->rows));
    p->part_steps = std::max<int64_t>(4, (p->steps + wanted - 1) / wanted);
    p->parts = (p->steps + p->part_steps - 1) / p->part_steps;
    auto up = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    p->stats = 0;
    p->tops = up(8 * (p->rows + 8 * kCUs));       // (parts are at most 8 kCUs / rows + 1)
    p->total = p->tops + up(4 * p->rows * p->chunks);
    return true;
}

#define TRY(expr)                          \
    do {                                   \
        const mpcnn_status rc_ = (expr);   \
        if (rc_ != MPCNN_OK) return rc_;   \
    } while (0)

struct Call {
    const float* bias;
    const float* totals;
    const uint8_t* done;
    int64_t end, sequences, beams, width, classes;
    float* totals_out;
    int32_t *parents, *classes_out;
    uint8_t* done_out;
};

mpcnn_status check(const Call& c, Plan* p, bool columns = false)
{
    if (c.sequences < 0 || c.beams < 1 || c.width < 1 || c.classes < 1)
        return fail(MPCNN_EINVAL, "%lld sequences of %lld beams, %lld wanted, %lld classes", (long long)c.sequences, (long long)c.beams, (long long)c.width, (long long)c.classes);
    if (c.end < -1 || c.end >= c.classes || (c.done && c.end < 0)) return fail(MPCNN_EINVAL, "class %lld of %lld ends a sequence", (long long)c.end, (long long)c.classes);
    if (c.width > mpcnn::kMaxBeams || !make_plan(c.sequences, c.beams, c.classes, p, columns))
        return fail(MPCNN_EUNSUPPORTED, "%lld sequences of %lld beams, %lld wanted, %lld classes: at most %d beams, %lld of all sequences, %lld classes", (long long)c.sequences,
                    (long long)c.beams, (long long)c.width, (long long)c.classes, mpcnn::kMaxBeams, (long long)kMaxRows, (long long)kMaxClasses);
    if (c.sequences > 0 && (!c.totals || !c.totals_out || !c.parents || !c.classes_out)) return fail(MPCNN_EINVAL, "null argument");
    if (((uintptr_t)c.bias | (uintptr_t)c.totals | (uintptr_t)c.totals_out | (uintptr_t)c.parents | (uintptr_t)c.classes_out) % 4)
        return fail(MPCNN_EINVAL, "an address is no multiple of its element's size");
    return MPCNN_OK;
}

mpcnn::ClassScores scores_of(const void* x, int64_t x_pitch, const void* w, int64_t w_pitch, const float* bias, int64_t rows, int64_t features, int64_t classes, int dtype)
{
    return mpcnn::ClassScores{x, w, x_pitch, w_pitch, bias, rows, features, classes, dtype};
}

// Outputs and the workspace may not meet an input or each other
mpcnn_status apart(const Call& c, const Span& scores, const void* ws, size_t ws_bytes, size_t need)
{
    if (!ws) return fail(MPCNN_EINVAL, "null argument");
    if (ws_bytes < need) return fail(MPCNN_EWORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, need);
    if ((uintptr_t)ws & 255u) return fail(MPCNN_EINVAL, "workspace must be 256-byte aligned");
    const uint64_t rows = (uint64_t)(c.sequences * c.beams), best = (uint64_t)(c.sequences * c.width);
    const Span in[] = {scores, {(uintptr_t)c.bias, 4 * (uint64_t)c.classes}, {(uintptr_t)c.totals, 4 * rows}, {(uintptr_t)c.done, rows}};
    const Span out[] = {{(uintptr_t)ws, need}, {(uintptr_t)c.totals_out, 4 * best}, {(uintptr_t)c.parents, 4 * best}, {(uintptr_t)c.classes_out, 4 * best},
                        {(uintptr_t)c.done_out, best}};
    for (size_t i = 0; i < sizeof out / sizeof *out; ++i) {
        for (const Span& s : in)
            if (meet(out[i], s)) return fail(MPCNN_EINVAL, "an output or the workspace overlaps an input");
        for (size_t j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return fail(MPCNN_EINVAL, "two outputs, or one and the workspace, overlap");
    }
    return MPCNN_OK;
}

mpcnn::BeamArgs args_of(const Plan& p, const Call& c, const void* scores, int64_t pitch, char* ws)
{
    mpcnn::BeamArgs a{};
    a.scores = scores; a.pitch = pitch; a.totals = c.totals; a.done = c.done; a.end = (int)c.end;
    a.sequences = (int)c.sequences; a.beams = (int)c.beams; a.width = (int)c.width;
    a.V = (int)c.classes; a.chunks = (int)p.chunks; a.steps = (int)p.steps; a.parts = (int)p.parts; a.part_steps = (int)p.part_steps;
    a.stats = (float2*)(ws + p.stats); a.stat_pitch = p.parts; a.tops = (float*)(ws + p.tops);
    a.totals_out = c.totals_out; a.parents = c.parents; a.classes = c.classes_out; a.done_out = c.done_out;
    return a;
}

template <typename T>
mpcnn_status select(const Plan& p, const Call& c, const void* scores, int64_t pitch, char* ws, hipStream_t st)
{
    mpcnn::BeamArgs a = args_of(p, c, scores, pitch, ws);
    a.bias = c.bias;
    mpcnn::beam_stats_kernel<T><<<(unsigned)(p.rows * p.parts), 256, 0, st>>>(a);
    mpcnn::beam_pick_kernel<mpcnn::BeamRow<T>><<<(unsigned)c.sequences, mpcnn::kPickThreads, mpcnn::pick_bytes((int)c.width), st>>>(a);
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

int64_t row_bytes(const mpcnn::BeamState& s) { return (int64_t)(s.segments - 1) * s.segment + s.unit * s.units; }

mpcnn_status make_states(const mpcnn_beam_state* t, int count, int64_t sequences, int64_t beams, mpcnn_beam_states** out)
{
    std::unique_ptr<mpcnn_beam_states> l(new mpcnn_beam_states);
    const int64_t most = (int64_t)1 << 40;
    for (int i = 0; i < count; ++i) {
        const mpcnn_beam_state& s = t[i];
        if (s.unit_bytes < 0 || s.units < 0 || s.segments < 0 || s.unit_bytes > most || s.units > most || s.segments > most ||
            s.row_pitch < 0 || s.row_pitch > most || s.segment_pitch < 0 || s.segment_pitch > most)
            return fail(MPCNN_EINVAL, "state %d: a size is below zero or above 2^40", i);
        if (!s.unit_bytes || !s.units || !s.segments || !sequences) continue;
        if (s.unit_bytes > most / s.units) return fail(MPCNN_EINVAL, "state %d: a segment above 2^40 bytes", i);
        const int64_t segment = s.unit_bytes * s.units;
        if (!s.data_dev) return fail(MPCNN_EINVAL, "state %d: null address", i);
        if (s.segments > 1 && (s.segment_pitch < segment || s.segment_pitch > most / s.segments)) return fail(MPCNN_EINVAL, "state %d: segments overlap", i);
        const int64_t row = (s.segments - 1) * s.segment_pitch + segment;
        if (sequences * beams > 1 && s.row_pitch < row) return fail(MPCNN_EINVAL, "state %d: rows overlap", i);
        if (row > (int64_t)1 << 34 || (segment + 15) / 16 > ((int64_t)1 << 30) / s.segments) return fail(MPCNN_EUNSUPPORTED, "state %d: a row above 2^34 bytes", i);
        const Span held{(uintptr_t)s.data_dev, (uint64_t)((sequences * beams - 1) * s.row_pitch + row)};
        l->states.push_back(mpcnn::BeamState{(char*)s.data_dev, s.row_pitch, s.segment_pitch, s.unit_bytes, s.units, (unsigned)s.segments, 0});
        l->held.push_back(held);
    }
    // Two tensors may lie in turn in one buffer: rows of one pitch, the second's between the first's
    std::vector<size_t> order(l->held.size());
    std::iota(order.begin(), order.end(), (size_t)0);
    std::sort(order.begin(), order.end(), [&](size_t a, size_t b) { return l->held[a].at < l->held[b].at; });
    for (size_t i = 0; i < order.size(); ++i)
        for (size_t j = i + 1; j < order.size() && meet(l->held[order[i]], l->held[order[j]]); ++j) {
            const mpcnn::BeamState &p = l->states[order[i]], &q = l->states[order[j]];
            const int64_t from = p.row ? (int64_t)(l->held[order[j]].at - l->held[order[i]].at) % p.row : 0;
            if (p.row != q.row || from < row_bytes(p) || from + row_bytes(q) > p.row) return fail(MPCNN_EINVAL, "two states overlap in memory");
        }
    if (l->states.size() > 65535) return fail(MPCNN_EUNSUPPORTED, "%d states: at most 65535", count);
    l->count = (int)l->states.size();
    l->sequences = (int)sequences;
    l->beams = (int)beams;
    const size_t bytes = sizeof(mpcnn::BeamState) * l->states.size();
    mpcnn::BeamState* dev = nullptr;
    hipError_t e = hipGetDevice(&l->device);
    if (e == hipSuccess && bytes) e = hipMalloc((void**)&dev, bytes);
    if (e == hipSuccess && bytes) e = hipMemcpy(dev, l->states.data(), bytes, hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        (void)hipFree(dev);
        return fail(e == hipErrorOutOfMemory ? MPCNN_ENOMEM : MPCNN_EHIP, "list of %d states: %s", count, hipGetErrorString(e));
    }
    l->d_states = dev;
    *out = l.release();
    return MPCNN_OK;
}

template <int M>
void launch_reorder(const mpcnn::ReorderArgs& a, dim3 grid, hipStream_t st)
{
    mpcnn::beam_reorder_kernel<M><<<grid, 256, 0, st>>>(a);
}

}  // namespace

extern "C" {

size_t mpcnn_workspace_bytes_beam(int64_t sequences, int64_t beams, int64_t classes)
{
    Plan p;
    return make_plan(sequences, beams, classes, &p) ? p.total : 0;
}

mpcnn_status mpcnn_beam_select(const void* scores_dev, int64_t scores_pitch, const float* bias_dev, const float* totals_dev, const uint8_t* done_dev, int64_t end,
                               int64_t sequences, int64_t beams, int64_t width, int64_t classes, mpcnn_dtype dtype, float* totals_out_dev, int32_t* parents_dev,
                               int32_t* classes_dev, uint8_t* done_out_dev, void* ws_dev, size_t ws_bytes, void* hip_stream)
{
    const Call c{bias_dev, totals_dev, done_dev, end, sequences, beams, width, classes, totals_out_dev, parents_dev, classes_dev, done_out_dev};
    Plan p;
    TRY(check(c, &p));
    if (dtype != MPCNN_F32 && dtype != MPCNN_BF16) return fail(MPCNN_EINVAL, "unknown type %d", (int)dtype);
    const int64_t size = dtype == MPCNN_F32 ? 4 : 2;
    if (sequences > 0 && !scores_dev) return fail(MPCNN_EINVAL, "null argument");
    if (scores_pitch < classes || scores_pitch > kMostPitch) return fail(MPCNN_EINVAL, "a pitch of %lld with %lld classes", (long long)scores_pitch, (long long)classes);
    if ((uintptr_t)scores_dev % size) return fail(MPCNN_EINVAL, "an address is no multiple of its element's size");
    TRY(apart(c, mpcnn::rows_span(scores_dev, p.rows, classes, scores_pitch, size), ws_dev, ws_bytes, p.total));
    if (!sequences) return MPCNN_OK;
    return dtype == MPCNN_F32 ? select<float>(p, c, scores_dev, scores_pitch, (char*)ws_dev, (hipStream_t)hip_stream)
                              : select<mpcnn::bf16>(p, c, scores_dev, scores_pitch, (char*)ws_dev, (hipStream_t)hip_stream);
}

size_t mpcnn_workspace_bytes_class_beam(int64_t sequences, int64_t beams, int64_t features, int64_t classes, mpcnn_dtype dtype)
{
    Plan p;
    if ((dtype != MPCNN_F32 && dtype != MPCNN_BF16) || !make_plan(sequences, beams, classes, &p, true)) return 0;
    return mpcnn::class_scores_bytes(scores_of(nullptr, 0, nullptr, 0, nullptr, p.rows, features, classes, dtype));
}

mpcnn_status mpcnn_class_beam(const void* x_dev, int64_t x_pitch, const void* w_dev, int64_t w_pitch, const float* bias_dev, const float* totals_dev,
                              const uint8_t* done_dev, int64_t end, int64_t sequences, int64_t beams, int64_t width, int64_t features, int64_t classes,
                              mpcnn_dtype dtype, float* totals_out_dev, int32_t* parents_dev, int32_t* classes_dev, uint8_t* done_out_dev, void* ws_dev,
                              size_t ws_bytes, void* hip_stream)
{
    const Call c{bias_dev, totals_dev, done_dev, end, sequences, beams, width, classes, totals_out_dev, parents_dev, classes_dev, done_out_dev};
    Plan p;
    TRY(check(c, &p, true));
    if (features < 1) return fail(MPCNN_EINVAL, "%lld features", (long long)features);
    if (dtype != MPCNN_F32 && dtype != MPCNN_BF16) return fail(MPCNN_EINVAL, "unknown type %d", (int)dtype);
    if (!w_dev || (sequences > 0 && !x_dev)) return fail(MPCNN_EINVAL, "null argument");
    if (x_pitch < features || w_pitch < features || x_pitch > kMostPitch || w_pitch > kMostPitch)
        return fail(MPCNN_EINVAL, "pitches of %lld and %lld with %lld features", (long long)x_pitch, (long long)w_pitch, (long long)features);
    const int64_t size = dtype == MPCNN_F32 ? 4 : 2;
    if (((uintptr_t)x_dev | (uintptr_t)w_dev) % size) return fail(MPCNN_EINVAL, "an address is no multiple of its element's size");
    const mpcnn::ClassScores s = scores_of(x_dev, x_pitch, w_dev, w_pitch, bias_dev, p.rows, features, classes, dtype);
    const size_t need = mpcnn::class_scores_bytes(s);
    if (!need) return fail(MPCNN_EUNSUPPORTED, "%lld rows, %lld features, %lld classes", (long long)p.rows, (long long)features, (long long)classes);
    TRY(apart(c, mpcnn::rows_span(x_dev, p.rows, features, x_pitch, size), ws_dev, ws_bytes, need));
    const Span w = mpcnn::rows_span(w_dev, classes, features, w_pitch, size);
    for (const Span& o : {Span{(uintptr_t)ws_dev, need}, Span{(uintptr_t)totals_out_dev, 4 * (uint64_t)(sequences * width)}, Span{(uintptr_t)parents_dev, 4 * (uint64_t)(sequences * width)},
                          Span{(uintptr_t)classes_dev, 4 * (uint64_t)(sequences * width)}, Span{(uintptr_t)done_out_dev, (uint64_t)(sequences * width)}})
        if (meet(o, w)) return fail(MPCNN_EINVAL, "an output or the workspace overlaps an input");
    if (!sequences) return MPCNN_OK;
    const hipStream_t st = (hipStream_t)hip_stream;
    mpcnn::KeptScores kept{};
    TRY(mpcnn::class_scores(s, (char*)ws_dev, &kept, st));
    mpcnn::BeamArgs a = args_of(p, c, kept.scores, kept.row, (char*)ws_dev);
    a.parts = (int)kept.tiles; a.stats = kept.stats; a.stat_pitch = kept.stat_pitch; a.tops = nullptr;
    const unsigned groups = (unsigned)sequences;
    const size_t lds = mpcnn::pick_bytes((int)width);
    switch (mpcnn::kChunk / kept.tile) {
        case 1: mpcnn::beam_pick_kernel<mpcnn::BeamColumn<1>><<<groups, mpcnn::kPickThreads, lds, st>>>(a); break;
        case 2: mpcnn::beam_pick_kernel<mpcnn::BeamColumn<2>><<<groups, mpcnn::kPickThreads, lds, st>>>(a); break;
        case 4: mpcnn::beam_pick_kernel<mpcnn::BeamColumn<4>><<<groups, mpcnn::kPickThreads, lds, st>>>(a); break;
        default: mpcnn::beam_pick_kernel<mpcnn::BeamColumn<8>><<<groups, mpcnn::kPickThreads, lds, st>>>(a); break;
    }
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

mpcnn_status mpcnn_beam_states_create(const mpcnn_beam_state* states_host, int count, int64_t sequences, int64_t beams, mpcnn_beam_states** out)
{
    if (!out || (count > 0 && !states_host)) return fail(MPCNN_EINVAL, "null argument");
    *out = nullptr;
    if (count < 0 || sequences < 0 || beams < 1) return fail(MPCNN_EINVAL, "%d states, %lld sequences of %lld beams", count, (long long)sequences, (long long)beams);
    if (beams > mpcnn::kMaxBeams || sequences > kMaxRows / beams)
        return fail(MPCNN_EUNSUPPORTED, "%lld sequences of %lld beams: at most %d beams, %lld of all sequences", (long long)sequences, (long long)beams, mpcnn::kMaxBeams, (long long)kMaxRows);
    try {
        return make_states(states_host, count, sequences, beams, out);
    } catch (const std::bad_alloc&) {
        return fail(MPCNN_ENOMEM, "out of host memory");
    }
}

void mpcnn_beam_states_destroy(mpcnn_beam_states* list)
{
    if (!list) return;
    int dev = -1;
    const bool moved = hipGetDevice(&dev) == hipSuccess && dev != list->device && hipSetDevice(list->device) == hipSuccess;
    (void)hipFree(list->d_states);
    if (moved) (void)hipSetDevice(dev);
    delete list;
}

mpcnn_status mpcnn_beam_reorder(const mpcnn_beam_states* list, const int32_t* parents_dev, int64_t length, void* hip_stream)
{
    if (!list) return fail(MPCNN_EINVAL, "null list");
    if (!parents_dev && list->sequences) return fail(MPCNN_EINVAL, "null argument");
    if ((uintptr_t)parents_dev % 4) return fail(MPCNN_EINVAL, "an address is no multiple of its element's size");
    const Span parents{(uintptr_t)parents_dev, 4 * (uint64_t)list->sequences * (uint64_t)list->beams};
    for (const Span& s : list->held)
        if (meet(parents, s)) return fail(MPCNN_EINVAL, "the parents lie in one of the states");
    int dev = -1;
    HIP_TRY(hipGetDevice(&dev));
    if (dev != list->device) return fail(MPCNN_EINVAL, "the list is on device %d, the current device is %d", list->device, dev);
    int64_t most = 0;                      // 16-byte pieces of a row
    for (const mpcnn::BeamState& s : list->states) {
        const int64_t units = length >= 0 ? std::min<int64_t>(length, s.units) : s.units;
        most = std::max(most, (units * s.unit + 15) / 16 * s.segments);
    }
    if (!most || !list->sequences || list->beams < 2) return MPCNN_OK;
    mpcnn::ReorderArgs a{};
    a.states = list->d_states; a.parents = parents_dev; a.length = length < 0 ? -1 : length;
    a.sequences = list->sequences; a.beams = list->beams;
    // no more than 2^23 workgroups (a launch has less than 2^32 threads): the rest of the sequences, and of a row, is the same workgroups' again
    const int64_t most_groups = (int64_t)1 << 23;
    const int64_t y = std::min({(int64_t)list->sequences, (int64_t)65535, most_groups / list->count});
    const int64_t x = std::max<int64_t>(1, std::min<int64_t>((most + 255) / 256, most_groups / (y * list->count)));
    const dim3 grid((unsigned)x, (unsigned)y, (unsigned)list->count);
    const hipStream_t st = (hipStream_t)hip_stream;
    if (a.beams <= 4) launch_reorder<4>(a, grid, st);
    else if (a.beams <= 8) launch_reorder<8>(a, grid, st);
    else if (a.beams <= 16) launch_reorder<16>(a, grid, st);
    else if (a.beams <= 32) launch_reorder<32>(a, grid, st);
    else launch_reorder<64>(a, grid, st);
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

}  // extern "C"
