// Lists of gradient (and parameter) tensors: their norm, clipping, and the gradient step (see include/mpcnn.h, kernels_update.hpp).
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <iterator>
#include <limits>
#include <map>
#include <memory>
#include <new>
#include <utility>
#include <vector>

#include "kernels_update.hpp"
#include "status.hpp"

using mpcnn::fail;

struct mpcnn_grad_list {
    int device = -1;
    long total = 0;
    int stretches = 0;
    bool params = false;
    // The tensors in runs, in their order: none of a run shares memory with another of it that a call writes.  Each run's first stretch, and the last one's
    // end, for calls that write the gradients and for those that write the parameters (empty: all tensors are one run).
    std::vector<int> grad_runs, param_runs;
    std::vector<std::pair<uintptr_t, uintptr_t>> held;   // the tensors' memory: begins and ends, in order, none meeting the next
    mpcnn::Stretch* d_table = nullptr;   // and, behind it, the partial sums
    double* d_partial = nullptr;
};

namespace mpcnn {

bool rate_fits(double rate, double scale)
{
    return std::isfinite(scale) && std::isfinite(rate) && std::fabs(rate * scale) <= (double)std::numeric_limits<float>::max();
}

unsigned stretch_length(long total)
{
    const long each = (total / 4096 + kStretchLeast - 1) / kStretchLeast * kStretchLeast;
    return (unsigned)std::min<long>(kStretch, std::max<long>(kStretchLeast, each));
}

template <bool LONE>
static void launch_mode(const UpdateArgs& a, int mode, unsigned groups, hipStream_t st)
{
    constexpr int threads = LONE ? 1024 : 256;
    if (mode == kOnlyNorm) update_kernel<kOnlyNorm, LONE><<<1, threads, 0, st>>>(a);
    else if (mode == kClip) update_kernel<kClip, LONE><<<groups, threads, 0, st>>>(a);
    else update_kernel<kStep, LONE><<<groups, threads, 0, st>>>(a);
}

void launch_update(UpdateArgs a, int mode, long total, const int* starts, int runs, hipStream_t st)
{
    if (runs && mode != kOnlyNorm) {
        // tensors that share memory: the norm, then one run after the other
        const int groups = (int)std::min<long>(kNormParts, ((long)a.stretches + 3) / 4);
        a.parts = groups;
        norm_parts_kernel<<<(unsigned)groups, 256, 0, st>>>(a);
        const Stretch* const table = a.table;
        for (int i = 0; i < runs; ++i) {
            a.table = table + starts[i];
            a.stretches = starts[i + 1] - starts[i];
            launch_mode<false>(a, mode, (unsigned)std::min<long>(kNormParts, ((long)a.stretches + 3) / 4), st);
        }
        return;
    }
    if (total <= kLoneNumbers && a.stretches <= kLoneStretches) {
        launch_mode<true>(a, mode, 1, st);
        return;
    }
    const int groups = (int)std::min<long>(kNormParts, ((long)a.stretches + 3) / 4);
    a.parts = groups;
    norm_parts_kernel<<<(unsigned)groups, 256, 0, st>>>(a);
    launch_mode<false>(a, mode, (unsigned)groups, st);
}

}  // namespace mpcnn

namespace {

struct Range { uintptr_t at; uint64_t bytes; bool param; };

// Whether two ranges of one kind overlap (same[param]), and whether a gradient and a parameter do (mixed)
void overlap(std::vector<Range>& r, bool (&same)[2], bool* mixed)
{
    std::sort(r.begin(), r.end(), [](const Range& x, const Range& y) { return x.at < y.at; });
    uintptr_t end[2] = {0, 0};           // of what has begun so far, gradients and parameters
    same[0] = same[1] = *mixed = false;
    for (const Range& x : r) {
        same[x.param] = same[x.param] || x.at < end[x.param];
        *mixed = *mixed || x.at < end[!x.param];
        end[x.param] = std::max<uintptr_t>(end[x.param], x.at + x.bytes);
    }
}

// The ranges of a run so far, which do not overlap, by where they begin
struct Run {
    std::map<uintptr_t, uintptr_t> ends;
    // Whether a tensor at [at, end) has to begin a new run (and, if so, it has)
    bool cut(uintptr_t at, uintptr_t end)
    {
        const auto next = ends.lower_bound(at);
        const bool meets = (next != ends.end() && next->first < end) || (next != ends.begin() && std::prev(next)->second > at);
        if (meets) ends.clear();
        ends.emplace(at, end);
        return meets;
    }
};

bool known(int dtype) { return dtype == MPCNN_F32 || dtype == MPCNN_BF16; }
uint64_t size_of(int dtype) { return dtype == MPCNN_BF16 ? 2 : 4; }

mpcnn_status make_list(const mpcnn_tensor* t, int count, mpcnn_grad_list** out)
{
    std::vector<Range> ranges;
    int64_t total = 0;
    int with = 0, filled = 0;
    for (int i = 0; i < count; ++i) {
        if (t[i].n < 0 || t[i].n > ((int64_t)1 << 40)) return fail(MPCNN_EINVAL, "tensor %d: %lld numbers", i, (long long)t[i].n);
        if (!known(t[i].grad_dtype) || (t[i].param_dev && !known(t[i].param_dtype))) return fail(MPCNN_EINVAL, "tensor %d: unknown type", i);
        if (!t[i].n) continue;
        if (!t[i].grad_dev) return fail(MPCNN_EINVAL, "tensor %d: null gradient", i);
        const uint64_t gs = size_of(t[i].grad_dtype), ps = size_of(t[i].param_dtype);
        if ((uintptr_t)t[i].grad_dev % gs || (t[i].param_dev && (uintptr_t)t[i].param_dev % ps))
            return fail(MPCNN_EINVAL, "tensor %d: address is no multiple of its element's size", i);
        ++filled;
        total += t[i].n;
        if (total > (int64_t)1 << 40) return fail(MPCNN_EINVAL, "too many numbers: over 2^40");
        ranges.push_back({(uintptr_t)t[i].grad_dev, (uint64_t)t[i].n * gs, false});
        if (t[i].param_dev) {
            ++with;
            ranges.push_back({(uintptr_t)t[i].param_dev, (uint64_t)t[i].n * ps, true});
        }
    }
    if (with && with != filled) return fail(MPCNN_EINVAL, "%d of %d tensors have parameters: all or none", with, filled);
    bool same[2], mixed = false;
    overlap(ranges, same, &mixed);
    if (mixed) return fail(MPCNN_EINVAL, "a gradient and a parameter overlap in memory");
    const unsigned len = mpcnn::stretch_length((long)total);
    std::vector<mpcnn::Stretch> table;
    std::vector<int> runs[2];
    Run run[2];
    for (int i = 0; i < count; ++i) {
        for (int k = 0; k < 2 && t[i].n; ++k) {
            if (!same[k]) continue;
            const uintptr_t at = (uintptr_t)(k ? t[i].param_dev : t[i].grad_dev);
            const bool cut = run[k].cut(at, at + t[i].n * size_of(k ? t[i].param_dtype : t[i].grad_dtype));
            if (cut || runs[k].empty()) runs[k].push_back((int)table.size());
        }
        for (int64_t at = 0; at < t[i].n; at += len) {
            mpcnn::Stretch s{};
            s.grad = (char*)t[i].grad_dev + at * (int64_t)size_of(t[i].grad_dtype);
            s.grad_bf16 = t[i].grad_dtype == MPCNN_BF16;
            if (t[i].param_dev) {
                s.param = (char*)t[i].param_dev + at * (int64_t)size_of(t[i].param_dtype);
                s.param_bf16 = t[i].param_dtype == MPCNN_BF16;
            }
            s.n = (unsigned)std::min<int64_t>(len, t[i].n - at);
            table.push_back(s);
        }
    }
    for (int k = 0; k < 2; ++k)
        if (same[k]) runs[k].push_back((int)table.size());
    if (table.size() > (size_t)1 << 30) return fail(MPCNN_EINVAL, "too many tensors: %d", count);
    std::unique_ptr<mpcnn_grad_list> l(new mpcnn_grad_list);
    l->grad_runs = std::move(runs[0]);
    l->param_runs = std::move(runs[1]);
    for (const Range& r : ranges) {          // (sorted)
        if (!l->held.empty() && r.at <= l->held.back().second) l->held.back().second = std::max(l->held.back().second, r.at + r.bytes);
        else l->held.emplace_back(r.at, r.at + r.bytes);
    }
    l->total = (long)total;
    l->stretches = (int)table.size();
    l->params = with > 0;
    const size_t bytes = sizeof(mpcnn::Stretch) * table.size(), partial = sizeof(double) * mpcnn::kNormParts;
    static_assert(sizeof(mpcnn::Stretch) % sizeof(double) == 0, "the partial sums behind the table are aligned");
    char* dev = nullptr;
    hipError_t e = hipGetDevice(&l->device);
    if (e == hipSuccess) e = hipMalloc((void**)&dev, bytes + partial);
    if (e == hipSuccess && bytes) e = hipMemcpy(dev, table.data(), bytes, hipMemcpyHostToDevice);
    if (e != hipSuccess) {
        (void)hipFree(dev);
        return fail(e == hipErrorOutOfMemory ? MPCNN_ENOMEM : MPCNN_EHIP, "list of %d tensors: %s", count, hipGetErrorString(e));
    }
    l->d_table = (mpcnn::Stretch*)dev;
    l->d_partial = (double*)(dev + bytes);
    *out = l.release();
    return MPCNN_OK;
}

// Whether the fp64 number at `norm` lies in the tensors' memory, in part or whole
bool holds(const mpcnn_grad_list* l, const double* norm)
{
    const uintptr_t at = (uintptr_t)norm, end = at + sizeof *norm;
    const auto next = std::lower_bound(l->held.begin(), l->held.end(), at, [](const auto& r, uintptr_t x) { return r.second <= x; });
    return next != l->held.end() && next->first < end;
}

mpcnn_status update(const mpcnn_grad_list* l, int mode, double rate, double scale, double bound, double* norm, void* stream)
{
    if (!l) return fail(MPCNN_EINVAL, "null list");
    if (mode == mpcnn::kOnlyNorm && !norm) return fail(MPCNN_EINVAL, "null argument");
    if ((uintptr_t)norm % sizeof(double)) return fail(MPCNN_EINVAL, "norm's address is no multiple of its size");
    if (norm && holds(l, norm)) return fail(MPCNN_EINVAL, "norm lies in one of the tensors");
    if (!mpcnn::rate_fits(rate, scale)) return fail(MPCNN_EINVAL, "scale %g, rate %g", scale, rate);
    if (!(bound > 0.0)) return fail(MPCNN_EINVAL, "max_norm = %g", bound);
    if (mode == mpcnn::kStep && l->stretches && !l->params) return fail(MPCNN_EINVAL, "the list has no parameters");
    int dev = -1;
    HIP_TRY(hipGetDevice(&dev));
    if (dev != l->device) return fail(MPCNN_EINVAL, "the list is on device %d, the current device is %d", l->device, dev);
    mpcnn::UpdateArgs a{};
    a.table = l->d_table;
    a.stretches = l->stretches;
    a.partial = l->d_partial;
    a.norm = norm;
    a.scale = std::fabs(scale);
    a.bound = bound;
    a.rate = rate * scale;
    const std::vector<int>& runs = mode == mpcnn::kClip ? l->grad_runs : l->param_runs;
    mpcnn::launch_update(a, mode, l->total, runs.data(), runs.empty() ? 0 : (int)runs.size() - 1, (hipStream_t)stream);
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

}  // namespace

extern "C" {

mpcnn_status mpcnn_grad_list_create(const mpcnn_tensor* tensors_host, int count, mpcnn_grad_list** out)
{
    if (!out || (count > 0 && !tensors_host)) return fail(MPCNN_EINVAL, "null argument");
    if (count < 0) return fail(MPCNN_EINVAL, "count = %d", count);
    *out = nullptr;
    try {
        return make_list(tensors_host, count, out);
    } catch (const std::bad_alloc&) {
        return fail(MPCNN_ENOMEM, "out of host memory");
    }
}

void mpcnn_grad_list_destroy(mpcnn_grad_list* list)
{
    if (!list) return;
    int dev = -1;
    const bool moved = hipGetDevice(&dev) == hipSuccess && dev != list->device && hipSetDevice(list->device) == hipSuccess;
    (void)hipFree(list->d_table);
    if (moved) (void)hipSetDevice(dev);
    delete list;
}

mpcnn_status mpcnn_grad_norm(const mpcnn_grad_list* list, double grad_scale, double* norm_dev, void* hip_stream)
{
    return update(list, mpcnn::kOnlyNorm, 1.0, grad_scale, INFINITY, norm_dev, hip_stream);
}

mpcnn_status mpcnn_grad_clip(const mpcnn_grad_list* list, double max_norm, double* norm_dev, void* hip_stream)
{
    return update(list, mpcnn::kClip, 1.0, 1.0, max_norm, norm_dev, hip_stream);
}

mpcnn_status mpcnn_sgd_step_list(const mpcnn_grad_list* list, double lr, double grad_scale, double max_norm, double* norm_dev,
                                 void* hip_stream)
{
    return update(list, mpcnn::kStep, lr, grad_scale, max_norm, norm_dev, hip_stream);
}

}  // extern "C"
