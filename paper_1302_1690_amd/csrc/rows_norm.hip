// Root-mean-square norm of rows, its gradients, and rows in 8 bits (include/mpcnn.h, mpcnn_rows_norm and what follows): checks and launches.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "kernels_rows_norm.hpp"
#include "spans.hpp"
#include "status.hpp"

using mpcnn::fail;
using mpcnn::meet;
using mpcnn::Span;

namespace {

constexpr int64_t kMaxRows = 0x7fffffff, kMaxFeatures = 1 << 20, kMostPitch = (int64_t)1 << 40;
constexpr int kCUs = 256;
// Rows one after the other of a lone workgroup, which has its rows one at a time or several.  us a call, lone / with shares: 4 x 4096 bf16 12.3 / 14.2, 8 x 4096 14.8 / 14.3, 32 x 768 fp32 (4 rows
// at a time) 12.6 / 14.5, 64 x 768 20 / 14.8, 128 x 100 bf16 (16 at a time) 12.3 / 14.2, 256 x 100 20 / 14.3
constexpr int64_t kLoneTurns[2] = {4, 8};
constexpr int64_t kManyPieces = 1 << 21;

int64_t padded_of(int64_t features) { return (features + mpcnn::kBlock - 1) / mpcnn::kBlock * mpcnn::kBlock; }

// How many lanes share a row, and its pieces of 8 features a lane (0: no workgroup's registers hold the row).  A lane of 1024 has 128 registers, of 512 256: the
// backward pass keeps three matrices and two sums a feature.  3000 x 16000 bf16 gradients from 8 bits: 66 us a call, 103 where rows are read twice.
struct Shape { int lanes, pieces; };
constexpr Shape kForward[8] = {{16, 1}, {16, 2}, {64, 1}, {64, 2}, {256, 1}, {256, 2}, {1024, 1}, {1024, 2}};
constexpr Shape kBackward[8] = {{16, 1}, {16, 2}, {64, 1}, {64, 2}, {256, 1}, {256, 2}, {1024, 1}, {512, 4}};
Shape shape_of(int64_t features, bool backward)
{
    for (const Shape& s : backward ? kBackward : kForward)
        if (features <= 8 * s.lanes * s.pieces) return s;
    return Shape{1024, 0};
}
template <bool BACKWARD, int I = 0, typename F>
void with_shape(const Shape& s, F&& f)
{
    constexpr Shape is = (BACKWARD ? kBackward : kForward)[I];
    if (s.lanes == is.lanes && s.pieces == is.pieces) f(std::integral_constant<int, is.lanes>{}, std::integral_constant<int, is.pieces>{});
    else if constexpr (I + 1 < 8) with_shape<BACKWARD, I + 1>(s, f);
}
int64_t groups_of(int64_t rows, const Shape& s, int64_t most)
{
    const int64_t slots = mpcnn::threads_of(s.lanes) / s.lanes;
    return std::max<int64_t>(1, std::min((rows + slots - 1) / slots, most));
}
// Workgroups of a backward call, each of which leaves a share of dgain: one for a few rows (no shares to add up)
int64_t back_groups(int64_t rows, int64_t features)
{
    const Shape s = shape_of(features, true);
    const int64_t slots = mpcnn::threads_of(s.lanes) / s.lanes;
    if (rows <= kLoneTurns[slots > 1] * slots) return 1;
    return groups_of(rows, s, s.lanes > 256 ? kCUs : 3 * kCUs);
}

bool known(int dtype) { return dtype == MPCNN_F32 || dtype == MPCNN_BF16; }
int64_t size_of(int dtype) { return dtype == MPCNN_BF16 ? 2 : 4; }

mpcnn_status sizes(int64_t rows, int64_t features, int dtype)
{
    if (rows < 0 || features < 1) return fail(MPCNN_EINVAL, "%lld rows, %lld features", (long long)rows, (long long)features);
    if (!known(dtype)) return fail(MPCNN_EINVAL, "unknown type %d", dtype);
    if (rows > kMaxRows || features > kMaxFeatures)
        return fail(MPCNN_EUNSUPPORTED, "%lld rows, %lld features: at most %lld, %lld", (long long)rows, (long long)features, (long long)kMaxRows, (long long)kMaxFeatures);
    return MPCNN_OK;
}
mpcnn_status matrix(const char* name, const void* m, int64_t pitch, int64_t features, int dtype)
{
    if (!m) return MPCNN_OK;
    if (pitch < features || pitch > kMostPitch) return fail(MPCNN_EINVAL, "%s: a pitch of %lld with %lld features", name, (long long)pitch, (long long)features);
    if ((uintptr_t)m % size_of(dtype)) return fail(MPCNN_EINVAL, "%s: address is no multiple of its element's size", name);
    return MPCNN_OK;
}
// A packed matrix (NULL, or without values: none) -> what kernels see
mpcnn_status packed(const char* name, const mpcnn_packed* p, mpcnn::Packed* out)
{
    *out = mpcnn::Packed{};
    if (!p || !p->values_dev) return MPCNN_OK;
    if (!p->scales_dev) return fail(MPCNN_EINVAL, "%s: no scales", name);
    if (p->kind != MPCNN_I8 && p->kind != MPCNN_E4M3) return fail(MPCNN_EINVAL, "%s: unknown kind %d", name, p->kind);
    if ((uintptr_t)p->values_dev % 16) return fail(MPCNN_EINVAL, "%s: address is no multiple of 16", name);
    *out = mpcnn::Packed{(unsigned char*)p->values_dev, p->scales_dev, p->kind};
    return MPCNN_OK;
}
Span values_span(const mpcnn::Packed& p, int64_t rows, int64_t padded) { return Span{(uintptr_t)p.values, (uint64_t)(rows * padded)}; }
Span scales_span(const mpcnn::Packed& p, int64_t rows, int64_t padded) { return Span{(uintptr_t)p.scales, (uint64_t)(rows * (padded / mpcnn::kBlock))}; }

// Outputs may not meet inputs or each other; `same`: but an output may be exactly the matrix of an input (which is read before it is written, number by number)
template <size_t I, size_t O>
mpcnn_status apart(const Span (&in)[I], const Span (&out)[O], const bool (&same)[O][I])
{
    for (size_t i = 0; i < O; ++i) {
        for (size_t j = 0; j < I; ++j)
            if (meet(out[i], in[j]) && !same[i][j]) return fail(MPCNN_EINVAL, "an output or the workspace overlaps an input");
        for (size_t j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return fail(MPCNN_EINVAL, "two outputs, or one and the workspace, overlap");
    }
    return MPCNN_OK;
}

template <typename T>
void launch_norm(const mpcnn::NormArgs& a, hipStream_t st)
{
    const Shape s = shape_of(a.D, false);
    if (!s.pieces) {
        mpcnn::rows_norm_long_kernel<T><<<(unsigned)groups_of(a.rows, s, 2 * kCUs), 1024, 0, st>>>(a);
        return;
    }
    with_shape<false>(s, [&](auto lanes, auto pieces) {
        constexpr int L = decltype(lanes)::value, E = decltype(pieces)::value;
        mpcnn::rows_norm_kernel<T, L, E><<<(unsigned)groups_of(a.rows, s, L > 256 ? 2 * kCUs : 8 * kCUs), mpcnn::threads_of(L), 0, st>>>(a);
    });
}
template <typename T, bool PACKED>
void launch_norm_back(const mpcnn::NormBackArgs& a, unsigned groups, hipStream_t st)
{
    const Shape s = shape_of(a.D, true);
    if (!s.pieces) {
        mpcnn::rows_norm_back_long_kernel<T, PACKED><<<groups, 1024, 0, st>>>(a);
        return;
    }
    with_shape<true>(s, [&](auto lanes, auto pieces) {
        constexpr int L = decltype(lanes)::value, E = decltype(pieces)::value;
        mpcnn::rows_norm_back_kernel<T, L, E, PACKED><<<groups, mpcnn::threads_of(L), 0, st>>>(a);
    });
}

#define TRY(expr)                          \
    do {                                   \
        const mpcnn_status rc_ = (expr);   \
        if (rc_ != MPCNN_OK) return rc_;   \
    } while (0)

// Rows of a workgroup of the packing kernels: 2048 pieces of 8 features, or 256 where there are few (16384 x 200 fp32 4.8 us, with 2048 6.4), and no more workgroups than a launch has
int pack_rows(int64_t rows, int64_t padded)
{
    const int64_t pieces = rows * (padded / 8) >= kManyPieces ? 2048 : 256;
    return (int)std::max<int64_t>(std::max<int64_t>(1, pieces / (padded / 8)), (rows + (1 << 23) - 1) >> 23);
}

mpcnn_status pack(const void* x, void* out, int64_t pitch, int64_t rows, int64_t features, int dtype, const mpcnn_packed* of, void* stream)
{
    TRY(sizes(rows, features, dtype));
    const void* const m = x ? x : out;
    mpcnn::PackArgs a{};
    TRY(packed("packed rows", of, &a.packed));
    if (rows > 0 && (!m || !a.packed.values)) return fail(MPCNN_EINVAL, "null argument");
    TRY(matrix(x ? "x" : "out", m, pitch, features, dtype));
    if (!rows) return MPCNN_OK;
    a.x = x; a.x_pitch = pitch; a.out = out; a.out_pitch = pitch; a.rows = rows; a.D = (int)features; a.padded = (int)padded_of(features);
    const Span span = mpcnn::rows_span(m, rows, features, pitch, size_of(dtype)), values = values_span(a.packed, rows, a.padded), scales = scales_span(a.packed, rows, a.padded);
    if (meet(span, values) || meet(span, scales) || (x && meet(values, scales))) return fail(MPCNN_EINVAL, "an output overlaps an input or another one");
    a.each = pack_rows(rows, a.padded);
    const unsigned groups = (unsigned)((rows + a.each - 1) / a.each);
    const hipStream_t st = (hipStream_t)stream;
    if (x && dtype == MPCNN_F32) mpcnn::rows_pack8_kernel<float><<<groups, 256, 0, st>>>(a);
    else if (x) mpcnn::rows_pack8_kernel<mpcnn::bf16><<<groups, 256, 0, st>>>(a);
    else if (dtype == MPCNN_F32) mpcnn::rows_unpack8_kernel<float><<<groups, 256, 0, st>>>(a);
    else mpcnn::rows_unpack8_kernel<mpcnn::bf16><<<groups, 256, 0, st>>>(a);
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

}  // namespace

extern "C" {

mpcnn_status mpcnn_rows_norm(const void* x_dev, int64_t x_pitch, const void* residual_dev, int64_t residual_pitch, const float* gain_dev, int64_t rows,
                             int64_t features, mpcnn_dtype dtype, double eps, void* y_dev, int64_t y_pitch, const mpcnn_packed* y_packed, void* h_dev,
                             int64_t h_pitch, const mpcnn_packed* h_packed, float* rstd_dev, void* hip_stream)
{
    TRY(sizes(rows, features, dtype));
    if (!(eps >= 0.0) || !std::isfinite((float)eps)) return fail(MPCNN_EINVAL, "eps = %g", eps);
    mpcnn::NormArgs a{};
    TRY(packed("y", y_packed, &a.y_packed));
    TRY(packed("h", h_packed, &a.h_packed));
    if (!gain_dev || (rows > 0 && !x_dev)) return fail(MPCNN_EINVAL, "null argument");
    TRY(matrix("x", x_dev, x_pitch, features, dtype));
    TRY(matrix("residual", residual_dev, residual_pitch, features, dtype));
    TRY(matrix("y", y_dev, y_pitch, features, dtype));
    TRY(matrix("h", h_dev, h_pitch, features, dtype));
    if (((uintptr_t)gain_dev | (uintptr_t)rstd_dev) % 4) return fail(MPCNN_EINVAL, "an address is no multiple of its element's size");
    const int64_t padded = padded_of(features), size = size_of(dtype);
    auto span = [&](const void* m, int64_t pitch) { return mpcnn::rows_span(m, rows, features, pitch, size); };
    const Span in[] = {span(x_dev, x_pitch), span(residual_dev, residual_pitch), {(uintptr_t)gain_dev, 4 * (uint64_t)features}};
    const Span out[] = {span(y_dev, y_pitch), span(h_dev, h_pitch), {(uintptr_t)rstd_dev, 4 * (uint64_t)rows}, values_span(a.y_packed, rows, padded),
                        scales_span(a.y_packed, rows, padded), values_span(a.h_packed, rows, padded), scales_span(a.h_packed, rows, padded)};
    auto is = [&](const void* o, int64_t o_pitch, const void* i, int64_t i_pitch) { return o == i && (o_pitch == i_pitch || rows < 2); };
    const bool same[7][3] = {{is(y_dev, y_pitch, x_dev, x_pitch), is(y_dev, y_pitch, residual_dev, residual_pitch), false},
                             {is(h_dev, h_pitch, x_dev, x_pitch), is(h_dev, h_pitch, residual_dev, residual_pitch), false}};
    TRY(apart(in, out, same));
    if (!rows) return MPCNN_OK;
    a.x = x_dev; a.x_pitch = x_pitch; a.residual = residual_dev; a.residual_pitch = residual_pitch; a.gain = gain_dev;
    a.rows = rows; a.D = (int)features; a.padded = (int)padded; a.eps = (float)eps;
    a.y = y_dev; a.y_pitch = y_pitch; a.h = h_dev; a.h_pitch = h_pitch; a.rstd = rstd_dev;
    if (dtype == MPCNN_F32) launch_norm<float>(a, (hipStream_t)hip_stream);
    else launch_norm<mpcnn::bf16>(a, (hipStream_t)hip_stream);
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

size_t mpcnn_workspace_bytes_norm(int64_t rows, int64_t features)
{
    if (rows < 0 || rows > kMaxRows || features < 1 || features > kMaxFeatures) return 0;
    return (size_t)((back_groups(rows, features) * features * 4 + 255) / 256 * 256);
}

mpcnn_status mpcnn_rows_norm_backward(const void* dy_dev, int64_t dy_pitch, const void* h_dev, int64_t h_pitch, const mpcnn_packed* h_packed,
                                      const float* gain_dev, const float* rstd_dev, const void* dh_dev, int64_t dh_pitch, int64_t rows, int64_t features,
                                      mpcnn_dtype dtype, void* dx_dev, int64_t dx_pitch, float* dgain_dev, void* ws_dev, size_t ws_bytes, void* hip_stream)
{
    TRY(sizes(rows, features, dtype));
    mpcnn::NormBackArgs a{};
    TRY(packed("h", h_packed, &a.h_packed));
    if (h_dev && a.h_packed.values) return fail(MPCNN_EINVAL, "h is given twice");
    if (!gain_dev || !ws_dev || (rows > 0 && (!dy_dev || !rstd_dev || (!h_dev && !a.h_packed.values)))) return fail(MPCNN_EINVAL, "null argument");
    TRY(matrix("dy", dy_dev, dy_pitch, features, dtype));
    TRY(matrix("h", h_dev, h_pitch, features, dtype));
    TRY(matrix("dh", dh_dev, dh_pitch, features, dtype));
    TRY(matrix("dx", dx_dev, dx_pitch, features, dtype));
    if (((uintptr_t)gain_dev | (uintptr_t)rstd_dev | (uintptr_t)dgain_dev) % 4) return fail(MPCNN_EINVAL, "an address is no multiple of its element's size");
    const size_t need = mpcnn_workspace_bytes_norm(rows, features);
    if (ws_bytes < need) return fail(MPCNN_EWORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, need);
    if ((uintptr_t)ws_dev & 255u) return fail(MPCNN_EINVAL, "workspace must be 256-byte aligned");
    const int64_t padded = padded_of(features), size = size_of(dtype);
    auto span = [&](const void* m, int64_t pitch) { return mpcnn::rows_span(m, rows, features, pitch, size); };
    const Span in[] = {span(dy_dev, dy_pitch), span(dh_dev, dh_pitch), span(h_dev, h_pitch), values_span(a.h_packed, rows, padded), scales_span(a.h_packed, rows, padded),
                       {(uintptr_t)gain_dev, 4 * (uint64_t)features}, {(uintptr_t)rstd_dev, 4 * (uint64_t)rows}};
    const Span out[] = {span(dx_dev, dx_pitch), {(uintptr_t)dgain_dev, 4 * (uint64_t)features}, {(uintptr_t)ws_dev, need}};
    auto is = [&](const void* i, int64_t pitch) { return dx_dev == i && (dx_pitch == pitch || rows < 2); };
    const bool same[3][7] = {{is(dy_dev, dy_pitch), is(dh_dev, dh_pitch), is(h_dev, h_pitch)}};
    TRY(apart(in, out, same));
    if (!dx_dev && !dgain_dev) return MPCNN_OK;
    const int groups = rows ? (int)back_groups(rows, features) : 0;
    a.dy = dy_dev; a.dy_pitch = dy_pitch; a.h = h_dev; a.h_pitch = h_pitch; a.dh = dh_dev; a.dh_pitch = dh_pitch;
    a.gain = gain_dev; a.rstd = rstd_dev; a.rows = rows; a.D = (int)features; a.padded = (int)padded; a.dx = dx_dev; a.dx_pitch = dx_pitch;
    if (dgain_dev) a.part = groups == 1 ? dgain_dev : (float*)ws_dev;
    const hipStream_t st = (hipStream_t)hip_stream;
    if (rows) {
        if (dtype == MPCNN_F32) a.h ? launch_norm_back<float, false>(a, (unsigned)groups, st) : launch_norm_back<float, true>(a, (unsigned)groups, st);
        else a.h ? launch_norm_back<mpcnn::bf16, false>(a, (unsigned)groups, st) : launch_norm_back<mpcnn::bf16, true>(a, (unsigned)groups, st);
    }
    if (dgain_dev && groups != 1)
        mpcnn::norm_gain_kernel<<<(unsigned)((features + mpcnn::kGainColumns - 1) / mpcnn::kGainColumns), mpcnn::kGainColumns * mpcnn::kGainStretches, 0, st>>>(
            (const float*)ws_dev, groups, (int)features, dgain_dev);
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

mpcnn_status mpcnn_rows_pack(const void* x_dev, int64_t x_pitch, int64_t rows, int64_t features, mpcnn_dtype dtype, const mpcnn_packed* out, void* hip_stream)
{
    if (rows > 0 && !x_dev) return fail(MPCNN_EINVAL, "null argument");
    return x_dev ? pack(x_dev, nullptr, x_pitch, rows, features, dtype, out, hip_stream) : sizes(rows, features, dtype);
}

mpcnn_status mpcnn_rows_unpack(const mpcnn_packed* x, int64_t rows, int64_t features, mpcnn_dtype dtype, void* out_dev, int64_t out_pitch, void* hip_stream)
{
    return pack(nullptr, out_dev, out_pitch, rows, features, dtype, x, hip_stream);
}

}  // extern "C"
