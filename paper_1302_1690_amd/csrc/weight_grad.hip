// The gradient of a linear layer's weights from rows kept in 8 bits (include/mpcnn.h, mpcnn_rows_weight_grad): the plan, checks and launches.
#include <algorithm>
#include <atomic>
#include <cstdint>

#include "kernels_weight_grad.hpp"
#include "spans.hpp"
#include "status.hpp"

using mpcnn::fail;
using mpcnn::meet;
using mpcnn::Span;

namespace {

constexpr int64_t kMaxRows = 0x7fffffff - 64, kMaxFeatures = 1 << 20, kMostPitch = (int64_t)1 << 40;
constexpr int64_t kMostResults = (int64_t)1 << 37;     // tiles of 128 x 128: 2^23 workgroups (a launch has less than 2^32 threads)
constexpr int64_t kPartRoom = (int64_t)256 << 20, kMostParts = 64;     // bytes of the partial sums, and how many
constexpr int kCUs = 256;
// Rows of bf16 that are no whole 16-byte pieces are copied into such where that is little beside the products.  us a call, copied / as they are, rows x outputs x features:
// 8192 x 4095 x 4096 int8 325 / 390, 4096 x 1001 x 300 30 / 29, 400 x 1001 x 1000 21 / 16, 4096 x 1001 x 100 28 / 22.
constexpr int64_t kAlignRows = 2048, kAlignFeatures = 1024;

int64_t padded_of(int64_t features) { return (features + mpcnn::kBlock - 1) / mpcnn::kBlock * mpcnn::kBlock; }

struct Plan { bool big, align; int tiles_m, tiles_n, blocks, splits, per_split; size_t part, total; };

// A tile's side, and what of its estimated time does not depend on the rows (make_plan)
struct Side {
    int64_t side, slots, tiles_m, tiles_n;
    double block_us, split_us;
    int64_t rounds(int64_t splits) const { return (tiles_m * tiles_n * splits + slots - 1) / slots; }
    // the operands' way for a row: every tile along one side reads the operand of the other
    double row_us(int64_t outs, int64_t features, bool f32) const { return ((f32 ? 4.0 : 2.0) * (double)(outs * tiles_n) + (double)(features * tiles_m)) * 1e-6 / 4.5; }
    double fixed(int64_t splits) const { return 1.5 * (double)rounds(splits) + (splits > 1 ? 6.0 + split_us * (double)splits : 0.0); }
};
Side side_of(bool big, int64_t outs, int64_t features, bool f32)
{
    Side s{};
    s.side = big ? 256 : 128; s.slots = big ? kCUs : 2 * kCUs;
    s.tiles_m = (outs + s.side - 1) / s.side; s.tiles_n = (features + s.side - 1) / s.side;
    s.block_us = f32 ? (big ? 2.8 : 2.3) : (big ? 2.0 : 1.3);
    s.split_us = 8e-6 * (double)outs * (double)features / 5.0;
    return s;
}
int64_t depth_of(bool f32) { return f32 ? 32 : 64; }
int64_t most_parts(int64_t blocks, int64_t outs, int64_t features) { return std::min({blocks, std::max<int64_t>(1, kPartRoom / (4 * outs * features)), kMostParts}); }
size_t part_bytes(int64_t splits, int64_t outs, int64_t features) { return splits > 1 ? (size_t)((4 * splits * outs * features + 255) / 256 * 256) : 0; }
bool copied(int64_t rows, int64_t outs, int64_t features, bool f32) { return !f32 && outs % 8 && rows >= kAlignRows && features >= kAlignFeatures; }
size_t copy_bytes(int64_t rows, int64_t outs) { return (size_t)(2 * rows * ((outs + 7) / 8 * 8)); }

// The most parts that so many blocks of rows, or fewer, are split into; it never falls when the blocks grow.  n parts take fixed(n) + max(products, operands) (make_plan), t parts, of tiles of the same side or of
// the other's, longer by less than block_us(t) rounds(t) (blocks / t + (t - 1) / t) - block_us(n) rounds(n) blocks / n in their products, and by the difference of the operands; both are linear in the blocks: where, at none
// and at so many, neither is more than fixed(n) - fixed(t), n is never taken.
int64_t most_splits(int64_t blocks, int64_t outs, int64_t features, bool f32)
{
    const int64_t most = most_parts(blocks, outs, features);
    double fixed[2][kMostParts + 1], share[2][kMostParts + 1], operands[2];      // share: of a block's products
    for (int big = 0; big < 2; ++big) {
        const Side s = side_of(big != 0, outs, features, f32);
        operands[big] = (double)depth_of(f32) * s.row_us(outs, features, f32);
        for (int64_t n = 1; n <= most; ++n) { fixed[big][n] = s.fixed(n); share[big][n] = s.block_us * (double)s.rounds(n) / (double)n; }
    }
    auto never = [&](int big, int64_t n) {
        for (int o = 0; o < 2; ++o)
            for (int64_t t = 1; t <= (o == big ? n - 1 : most); ++t) {
                const double saved = fixed[big][n] - fixed[o][t] - 1e-3;         // (more than estimates' roundings)
                if (saved >= share[o][t] * (double)(t - 1) + std::max(0.0, share[o][t] - share[big][n]) * (double)blocks && saved >= (operands[o] - operands[big]) * (double)blocks && saved >= 0.0)
                    return true;
            }
        return false;
    };
    int64_t n = most;
    while (n > 1 && never(0, n) && never(1, n)) --n;
    return n;
}
size_t most_bytes(int64_t rows, int64_t outs, int64_t features, bool f32)
{
    const int64_t blocks = std::max<int64_t>(1, (rows + depth_of(f32) - 1) / depth_of(f32));
    return part_bytes(most_splits(blocks, outs, features, f32), outs, features) + (copied(rows, outs, features, f32) ? copy_bytes(rows, outs) : 0);
}

// Tiles of 256 x 256 (a workgroup per compute unit) or of 128 x 128 (two), the rows whole or split: whichever should take least.  us a block of rows of a tile, measured (bf16 64
// rows, fp32 32): 256 x 256 2.0 and 2.8, two of 128 x 128 side by side 1.3 and 2.3; a split costs its sums' way to memory and back and a launch; operands come at 4.5 TB/s.  us a call, split / whole: 213 x 37 x 100 fp32
// 14 / 18.
bool make_plan(int64_t rows, int64_t outs, int64_t features, int dtype, Plan* p)
{
    if (rows < 0 || rows > kMaxRows || outs < 1 || outs > kMaxFeatures || features < 1 || features > kMaxFeatures || outs * features > kMostResults) return false;
    *p = Plan{};
    const bool f32 = dtype == MPCNN_F32;
    const int64_t blocks = std::max<int64_t>(1, (rows + depth_of(f32) - 1) / depth_of(f32)), most = most_parts(blocks, outs, features);
    p->blocks = (int)blocks;
    double least = 0.0;
    for (int big = 0; big < 2; ++big) {
        const Side s = side_of(big != 0, outs, features, f32);
        for (int64_t splits = 1; splits <= most; ++splits) {
            const int64_t each = (blocks + splits - 1) / splits;
            if (splits > 1 && (blocks + each - 1) / each != splits) continue;
            const double products = (double)s.rounds(splits) * s.block_us * (double)each, operands = (double)rows * s.row_us(outs, features, f32);
            const double us = s.fixed(splits) + std::max(products, operands);
            if (p->splits && us >= least) continue;
            least = us;
            p->big = big != 0; p->tiles_m = (int)s.tiles_m; p->tiles_n = (int)s.tiles_n; p->splits = (int)splits; p->per_split = (int)each;
        }
    }
    p->part = part_bytes(p->splits, outs, features);
    p->align = copied(rows, outs, features, f32);
    p->total = p->part + (p->align ? copy_bytes(rows, outs) : 0);
    return true;
}

template <typename T, int KIND, int WM, int WN, int MT, int NT, int KB, bool DIRECT>
mpcnn_status launch_instance(const mpcnn::WeightGradArgs& a, hipStream_t st)
{
    constexpr int lds = 2 * KB * 2 * 32 * ((sizeof(T) == 4 ? 3 : 1) * WM * MT + WN * NT);
    auto* kernel = &mpcnn::weight_grad_kernel<T, KIND, WM, WN, MT, NT, KB, DIRECT>;
    if constexpr (lds > 64 * 1024) {       // must be said once per device
        static std::atomic<uint64_t> said{0};
        int dev = 0;
        HIP_TRY(hipGetDevice(&dev));
        if (!(said.load(std::memory_order_relaxed) >> (dev & 63) & 1)) {
            HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
            said.fetch_or(1ull << (dev & 63), std::memory_order_relaxed);
        }
    }
    const int64_t all = (int64_t)a.tiles_m * a.tiles_n * a.splits;
    kernel<<<(unsigned)((all + 7) / 8 * 8), 64 * WM * WN, lds, st>>>(a);
    return MPCNN_OK;
}

template <typename T, int WM, int WN, int MT, int NT, int KB, bool DIRECT = false>
mpcnn_status launch(const mpcnn::WeightGradArgs& a, hipStream_t st)
{
    return a.x.kind == MPCNN_I8 ? launch_instance<T, MPCNN_I8, WM, WN, MT, NT, KB, DIRECT>(a, st) : launch_instance<T, MPCNN_E4M3, WM, WN, MT, NT, KB, DIRECT>(a, st);
}

}  // namespace

extern "C" {

size_t mpcnn_workspace_bytes_weight_grad(int64_t rows, int64_t outs, int64_t features, mpcnn_dtype dtype)
{
    Plan p;
    if ((dtype != MPCNN_F32 && dtype != MPCNN_BF16) || !make_plan(rows, outs, features, dtype, &p)) return 0;
    return std::max<size_t>(256, most_bytes(rows, outs, features, dtype == MPCNN_F32));
}

mpcnn_status mpcnn_rows_weight_grad(const void* dy_dev, int64_t dy_pitch, const mpcnn_packed* x, int64_t rows, int64_t outs, int64_t features, mpcnn_dtype dtype,
                                    void* dw_dev, mpcnn_dtype dw_dtype, void* ws_dev, size_t ws_bytes, void* hip_stream)
{
    if (rows < 0 || outs < 1 || features < 1) return fail(MPCNN_EINVAL, "%lld rows, %lld outputs, %lld features", (long long)rows, (long long)outs, (long long)features);
    if ((dtype != MPCNN_F32 && dtype != MPCNN_BF16) || (dw_dtype != MPCNN_F32 && dw_dtype != MPCNN_BF16))
        return fail(MPCNN_EINVAL, "unknown type %d or %d", (int)dtype, (int)dw_dtype);
    if (!dw_dev || !ws_dev || (rows > 0 && (!dy_dev || !x || !x->values_dev || !x->scales_dev))) return fail(MPCNN_EINVAL, "null argument");
    if (rows > 0 && x->kind != MPCNN_I8 && x->kind != MPCNN_E4M3) return fail(MPCNN_EINVAL, "unknown kind %d", x->kind);
    if (dy_pitch < outs || dy_pitch > kMostPitch) return fail(MPCNN_EINVAL, "a pitch of %lld with %lld outputs", (long long)dy_pitch, (long long)outs);
    const int64_t size = dtype == MPCNN_F32 ? 4 : 2, dw_size = dw_dtype == MPCNN_F32 ? 4 : 2;
    if ((uintptr_t)dy_dev % size || (uintptr_t)dw_dev % dw_size || (rows > 0 && (uintptr_t)x->values_dev % 16))
        return fail(MPCNN_EINVAL, "an address is no multiple of its element's size, or packed rows' none of 16");
    Plan p;
    if (!make_plan(rows, outs, features, dtype, &p))
        return fail(MPCNN_EUNSUPPORTED, "%lld rows, %lld outputs, %lld features: at most %lld, %lld, %lld, and %lld weights", (long long)rows, (long long)outs, (long long)features,
                    (long long)kMaxRows, (long long)kMaxFeatures, (long long)kMaxFeatures, (long long)kMostResults);
    if (ws_bytes < p.total) return fail(MPCNN_EWORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, p.total);
    if ((uintptr_t)ws_dev & 255u) return fail(MPCNN_EINVAL, "workspace must be 256-byte aligned");
    const int64_t padded = padded_of(features);
    const Span dw{(uintptr_t)dw_dev, (uint64_t)(outs * features * dw_size)}, ws{(uintptr_t)ws_dev, p.total}, dy = mpcnn::rows_span(dy_dev, rows, outs, dy_pitch, size);
    const Span values{rows > 0 ? (uintptr_t)x->values_dev : 0, (uint64_t)(rows * padded)}, scales{rows > 0 ? (uintptr_t)x->scales_dev : 0, (uint64_t)(rows * (padded / mpcnn::kBlock))};
    for (const Span& in : {dy, values, scales})
        if (meet(in, dw) || meet(in, ws)) return fail(MPCNN_EINVAL, "an output or the workspace overlaps an input");
    if (meet(dw, ws)) return fail(MPCNN_EINVAL, "the output and the workspace overlap");
    const hipStream_t st = (hipStream_t)hip_stream;
    const int64_t n = outs * features;
    const unsigned sum_groups = (unsigned)std::min<int64_t>(8192, (n + 63) / 64);
    if (!rows) {
        mpcnn::weight_grad_sum_kernel<<<sum_groups, 256, 0, st>>>(nullptr, 0, n, dw_dev, dw_dtype == MPCNN_BF16);
        HIP_TRY(hipGetLastError());
        return MPCNN_OK;
    }
    mpcnn::WeightGradArgs a{};
    a.dy = dy_dev; a.dy_pitch = dy_pitch; a.x = mpcnn::Packed{(unsigned char*)x->values_dev, x->scales_dev, x->kind};
    a.N = (int)rows; a.M = (int)outs; a.D = (int)features; a.padded = (int)padded;
    a.blocks = p.blocks; a.per_split = p.per_split; a.splits = p.splits; a.tiles_m = p.tiles_m; a.tiles_n = p.tiles_n;
    a.dw = dw_dev; a.dw_bf16 = dw_dtype == MPCNN_BF16;
    a.part = p.splits > 1 ? (float*)ws_dev : nullptr;
    // (a block's fetches are 32-bit offsets from its first row)
    auto whole = [](const void* m, int64_t pitch, int64_t columns) { return (uintptr_t)m % 16 == 0 && pitch % 8 == 0 && columns % 8 == 0 && pitch * 128 < (1ll << 31); };
    mpcnn_status rc;
    if (dtype == MPCNN_F32) {
        rc = p.big ? launch<float, 2, 4, 4, 2, 32>(a, st) : launch<float, 2, 2, 2, 2, 32>(a, st);
    } else {
        const int64_t aligned = (outs + 7) / 8 * 8;
        int64_t columns = outs;
        if (p.align) {
            mpcnn::bf16* const to = (mpcnn::bf16*)((char*)ws_dev + p.part);
            const int64_t pieces = rows * (aligned / 8);
            mpcnn::weight_grad_align_kernel<<<(unsigned)std::min<int64_t>(8192, (pieces + 255) / 256), 256, 0, st>>>((const mpcnn::bf16*)dy_dev, dy_pitch, rows, (int)outs, to, (int)aligned);
            a.dy = to; a.dy_pitch = columns = aligned;
        }
        a.dy_bytes = ((rows - 1) * a.dy_pitch + columns) * 2;
        const bool direct = whole(a.dy, a.dy_pitch, columns);
        rc = p.big && direct ? launch<mpcnn::bf16, 2, 4, 4, 2, 64, true>(a, st)
             : p.big         ? launch<mpcnn::bf16, 2, 4, 4, 2, 64>(a, st)
             : direct        ? launch<mpcnn::bf16, 2, 2, 2, 2, 64, true>(a, st)
                             : launch<mpcnn::bf16, 2, 2, 2, 2, 64>(a, st);
    }
    if (rc != MPCNN_OK) return rc;
    if (p.splits > 1) mpcnn::weight_grad_sum_kernel<<<sum_groups, 256, 0, st>>>(a.part, p.splits, n, dw_dev, a.dw_bf16);
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

}  // extern "C"
