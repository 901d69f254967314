// The class layer on rows of features with its softmax cross-entropy and its gradients, for label sets of any size (see include/mpcnn.h,
// mpcnn_class_loss and mpcnn_class_backward): the plan, the workspace and the launches.
//
//   scores s[v][n] = w[v] . x[n] + bias[v],  lse[n] = log sum_v exp s[v][n],  loss[n] = weight[n] (lse[n] - s[label[n]][n])
//   delta[n][v] = exp(s[v][n] - lse[n]) - [v = label[n]]
//   dx[n] = weight[n] sum_v delta[n][v] w[v],   dw[v] = sum_n weight[n] delta[n][v] x[n],   db[v] = sum_n weight[n] delta[n][v]
//
// The classes are taken in pieces.  A first round over them leaves, per row, each tile's largest score and sum of exponentials, and no scores.
// The second computes a piece's scores again, as the derivative, which it multiplies with the weights and the features
// (kernels_rows_product.hpp).  Where the scores of all classes fit the room that a piece's take (kRoom) and are more work than traffic
// (kKeepFeatures), they are kept from the first round.
#include <algorithm>
#include <atomic>
#include <cstdint>

#include "class_scores.hpp"
#include "kernels_rows_direct.hpp"
#include "rows_few.hpp"
#include "kernels_rows_parts.hpp"
#include "kernels_rows_product.hpp"
#include "spans.hpp"
#include "status.hpp"

using mpcnn::fail;
using mpcnn::meet;
using mpcnn::Span;

namespace {

constexpr int64_t kMaxRows = 1 << 20, kMaxFeatures = 1 << 20, kMaxClasses = 0x7fffffff - 1024;   // (32-bit offsets inside a tile)
constexpr int64_t kRoom = (int64_t)1 << 28;            // derivatives of a piece: 0.5 GB (1 GB with fp32 storage), and scores that are kept: 1 GB
// Scores that fit are kept where computing them again takes longer than their way to memory and back: with so many features and more, fp32 and
// bf16.  us, kept / computed again: 8000 x 8000 with 64 features 375 / 349 and 267 / 219, with 128 405 / 410 and 290 / 242, with 256
// 536 / 564 and 335 / 301, with 512 770 / 874 and 423 / 433, with 1024 1233 / 1467 and 544 / 605; 12000 x 20000 with 256 1676 / 1737 and 996 / 915,
// with 1024 4351 / 5288 and 2077 / 2284; 4000 x 4000 with 64 168 / 169 and 132 / 131.
constexpr int kKeepFeatures[2] = {128, 512};
constexpr int64_t kWeightRoom = (int64_t)512 << 20;    // bytes of a piece's class weights, brought into blocks
constexpr int64_t kPartRoom = (int64_t)256 << 20;      // bytes of a product's partial sums
constexpr int kMaxPiece = 1 << 20;
constexpr int kCUs = 256;
// A launch has less than 2^32 threads (of workgroups of 256: less than kMostGroups of them) and its grid's second side less than 2^16.  Products of this many
// results stay below that with tiles of either size (128 x 128: half of it).
constexpr int64_t kMostGroups = 1 << 24, kMostSide = (1 << 16) - 1, kMostResults = (int64_t)1 << 37;

inline int64_t up_to(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

struct Tiling { bool big; int tiles_m, tiles_n, splits, per_split; };

// Tiles of 256 x 256 (a workgroup per compute unit) or of 128 x 128 (two), the sum over k whole or split so that the parts fill one to four
// rounds of workgroups: whichever should take least.  A step of k (128 bytes of a row) of a tile takes 1.9 us (measured: 1.15 PFLOP/s on
// 256 x 256) or, two side by side, 1.3; fp32 storage's steps half as long again; a split costs the partial sums' way to memory and
// back (12 bytes of traffic at 5 TB/s each) and a launch.
Tiling tiling_of(int64_t M, int64_t N, int64_t blocks, int64_t most_splits, bool halves)
{
    M = std::max<int64_t>(M, 1); N = std::max<int64_t>(N, 1);   // (no rows: nothing is launched)
    Tiling best{};
    double least = 0.0;
    for (int big = 0; big < 2; ++big) {
        const int64_t side = big ? 256 : 128, slots = big ? kCUs : 2 * kCUs;
        const int64_t tiles = (M + side - 1) / side * ((N + side - 1) / side);
        for (int round = 0; round <= 4; ++round) {
            const int64_t splits = round ? std::min({round * slots / tiles, most_splits, blocks / 4}) : 1;
            if (round && splits < 2) continue;
            Tiling t{};
            t.big = big != 0;
            t.tiles_m = (int)((M + side - 1) / side);
            t.tiles_n = (int)((N + side - 1) / side);
            t.per_split = (int)((blocks + splits - 1) / splits);
            t.splits = (int)((blocks + t.per_split - 1) / t.per_split);
            const int64_t rounds = (tiles * t.splits + slots - 1) / slots;
            const double us = (double)rounds * (3.0 + t.per_split * (big ? 1.9 : 1.3) * (halves ? 1.5 : 1.0)) +
                              (t.splits > 1 ? 4.0 + 12e-6 * (double)M * (double)N * t.splits / 5.0 : 0.0);
            if (!best.splits || us < least) { best = t; least = us; }
        }
    }
    return best;
}

// Two to six launches (kernels_rows_direct.hpp) instead of a dozen: up to this much work, rows x features x classes, and up to more with few rows.
// Microseconds a call, in few launches / as much work, fp32 and bf16: gradients of 1000 x 1000 x 1000 (1e9) 109 / 114 and 63 / 73, of 1000 x 200 x 1000 (2e8) 49 / 88 and 34 / 68,
// of 3000 x 500 x 1000 (1.5e9) 154 / 120 and 90 / 77; the loss of 1000 x 1000 x 2000 (2e9) 66 / 55 and 34 / 33, of 4000 x 2000 x 200
// (1.6e9) 62 / 78 and 40 / 46; gradients of 20 x 4000 x 20000 (1.6e9) 336 / 586 and 170 / 274, of 40 x 1000 x 100000 (4e9) 699 / 818
// and 382 / 374, of 64 x 4096 x 8000 (2e9) 203 / 335 and 149 / 124.
constexpr int64_t kDirectWork = 1200000000, kDirectLossWork = 2000000000, kDirectFewRows = 64, kDirectFewWork[2] = {4000000000, 1600000000};

// Classes from which on gradients are rows_few_grads', of up to 4 rows and of up to 16.  us a call, there / in tiles (kernels_rows_direct.hpp), fp32 and bf16:
// 4 x 1000 x 512 27 / 25 and 27 / 24, x 1024 28 / 29 and 27 / 28, x 2048 30 / 35 and 27 / 30; 5 x 1000 x 4096 38 / 39 and 33 / 32, 8 x 1000 x 2048 36 / 36 and 29 / 30,
// x 4096 47 / 40 and 38 / 32, x 8192 54 / 51 and 39 / 41, x 16384 69 / 74 and 44 / 58; 12 x 200 x 4096 28 / 31 and 27 / 30; 16 x 1000 x 4096 47 / 40 and 44 / 33, x 16384 69 / 74
// and 56 / 59; 16 x 4096 x 4096 81 / 87 and 65 / 68.  And classes from which on scores are rows_few_scores': the first of up to 3 fp32 rows, the second of more, and of up to
// 2 bf16 rows (times in kernels_rows_few.hpp).
constexpr int64_t kFewClasses[2] = {1024, 4096}, kFewScoreClasses[2] = {1024, 24576};

// bf16 class weights from which on the scores of up to 4 and of up to 12 rows are the vector ALU's, too (fewer come from the last-level cache fast enough;
// times in kernels_rows_few.hpp)
constexpr int64_t kFewWeights[2] = {70000000, 150000000};

// fp32 class weights from which on the scores of 9 to so many rows are rows_wide_scores_kernel's (but for those that are rows_few_scores').  us a call of the
// loss, with it / without (rows_direct_scores or, with more work, weights brought into blocks): 16 x 4096 x 50000 260 / 455, 32 x 4096 x 50000 265 / 870,
// 64 x 4096 x 50000 310 / 860, 100 x 4096 x 20000 225 / 320, 128 x 4096 x 50000 538 / 894, 32 x 1000 x 20000 44 / 47, 64 x 1000 x 20000 57 / 68,
// 32 x 4096 x 3000 50 / 65, 64 x 4096 x 3000 58 / 66, 64 x 1000 x 5000 38 / 37.
constexpr int64_t kWideRows = 128, kWideWeights = 12000000;

struct Plan {
    bool halves, train, keep, direct, few, few_scores, wide;
    int grad_groups;                     // few: workgroups along the classes,
    int64_t score_each, grad_each;       // their classes, and those of the scores' workgroups
    int score_deal, score_v, score_n;    // direct: waves that share a tile's sum, tiles along classes and rows
    struct { int deal, m, along, splits, each; } gx, gw;   // of the gradients: tiles along rows or classes and along features, parts of the sum, their length
    int N, D;
    int64_t V, Np;                       // Np: rows, padded to whole blocks
    int64_t d_bytes, n_bytes;            // a row of blocks along the features, along the rows
    int64_t piece, most_piece;           // classes; where the class weights are read as they are and no derivative is kept
    int64_t stat_tiles;
    Tiling dx, dw;                       // of a whole piece
    Tiling sc;                           // of the scores, where there is one piece
    size_t peaks, stats, label_score, lse, weight, loss_part, x_rows, x_cols, w_rows, x_split, score, score_part, delta, db_part,
        dx_part, dw_part, total;
    int64_t bytes_along(int64_t n) const { return halves ? up_to(n, 32) * 4 : up_to(n, 64) * 2; }
    int64_t v_blocks(int64_t n) const { return (n + (halves ? 31 : 63)) / (halves ? 32 : 64); }   // of the sum over n classes
    bool dx_parts() const { return dx.splits > 1 || piece < V; }
};

// Whose the scores of little work are: rows_wide_scores_kernel's, rows_few_scores_kernel's, or rows_direct_scores_kernel's
bool wide_scores(bool halves, int64_t rows, int64_t features, int64_t classes)
{
    return halves && rows > 8 && rows <= kWideRows && classes >= kWideWeights / features && (rows > mpcnn::kFewScoreRows || classes < kFewScoreClasses[1]);
}
bool few_scores(bool halves, int64_t rows, int64_t features, int64_t classes)
{
    if (halves) return rows <= mpcnn::kFewScoreRows && classes >= kFewScoreClasses[rows <= 3 ? 0 : 1];
    if (rows <= 2) return classes >= kFewScoreClasses[1];
    return rows <= mpcnn::kFewScoreRows && classes >= kFewWeights[rows <= 4 ? 0 : 1] / features;
}
int64_t score_groups(bool wide, int64_t rows, int64_t classes)
{
    return wide ? (classes + 31) / 32 * (rows <= 32 ? 1 : up_to(rows, 64) / 64) : (classes + 63) / 64;
}
// a tile of 32 x 32 for four waves, one of 64 x 64 where that gives every compute unit two workgroups or the sum has one step
int deal_of(int64_t m, int64_t n, int64_t k) { return (m + 63) / 64 * ((n + 63) / 64) >= 2 * kCUs || k <= mpcnn::kDirectK ? 1 : 4; }
int dealt_tiles(int64_t n, int deal) { return (int)((n + (deal == 4 ? 31 : 63)) / (deal == 4 ? 32 : 64)); }
void plan_scores(Plan* p, int64_t rows, int64_t features, int64_t classes)
{
    p->score_deal = deal_of(classes, rows, features);
    p->score_v = dealt_tiles(classes, p->score_deal); p->score_n = dealt_tiles(rows, p->score_deal);
    if (p->wide) p->score_v = dealt_tiles(classes, 4);
    if (p->few_scores) {
        const int64_t round = mpcnn::kFewRound;
        p->score_each = ((classes + round - 1) / round + 8 * kCUs - 1) / (8 * kCUs) * round;   // whole rounds
        p->score_v = (int)((classes + p->score_each - 1) / p->score_each);
    }
}
int64_t x_split_bytes(int64_t rows, int64_t features) { return up_to(rows, rows <= 32 ? 32 : 64) * up_to(features, mpcnn::kDirectK) * 6; }

bool make_plan(int64_t rows, int64_t features, int64_t classes, int dtype, bool train, Plan* p)
{
    if (rows < 0 || rows > kMaxRows || features < 1 || features > kMaxFeatures || classes < 1 || classes > kMaxClasses) return false;
    *p = Plan{};
    p->halves = dtype == MPCNN_F32;
    p->train = train;
    p->N = (int)rows; p->D = (int)features; p->V = classes;
    p->Np = up_to(std::max<int64_t>(rows, 1), 64);
    p->d_bytes = p->bytes_along(features);
    p->n_bytes = p->bytes_along(p->Np);
    size_t at = 0;
    auto take = [&](int64_t bytes) { const size_t o = at; at += (size_t)up_to(bytes, 256); return o; };
    const bool fits = classes <= kRoom / p->Np;
    p->keep = train && fits && features >= kKeepFeatures[p->halves ? 0 : 1];
    const int64_t most = rows <= kDirectFewRows ? kDirectFewWork[p->halves ? 0 : 1] : train ? kDirectWork : kDirectLossWork;
    p->wide = wide_scores(p->halves, rows, features, classes);
    p->direct = (rows <= mpcnn::kFewRows || rows * classes <= most / features || (p->wide && !train)) && (fits || !train);
    // few rows and many classes: the gradients, and the scores of still fewer, on the vector ALU (kernels_rows_few.hpp has the times)
    p->few = p->direct && train && rows > 0 && rows <= mpcnn::kFewRows && classes >= kFewClasses[rows <= 4 ? 0 : 1];
    if (p->direct && rows > 0) p->few_scores = few_scores(p->halves, rows, features, classes);
    // what its launches cannot have is much work's, in pieces: 2^28 fp32 classes (of more than 64 rows; of more than 12, 2^29) or 2^30 bf16 ones, the
    // derivative of the last few of 2^22
    if (!p->few_scores && score_groups(p->wide, rows, classes) >= kMostGroups) p->direct = false;
    if (train && !p->few && (classes + mpcnn::kDeltaSide - 1) / mpcnn::kDeltaSide > kMostSide) p->direct = false;
    if (p->direct) {
        plan_scores(p, rows, features, classes);
        if (p->few) {
            // shares of dx: 512 workgroups, fewer where their shares' way to memory and back would be more than an eighth of the class weights' passes
            const int64_t each = mpcnn::few_columns((int)rows) * mpcnn::kFewThreads, along = (features + each - 1) / each;
            const int64_t by_traffic = classes * (p->halves ? 4 : 2) * 3 / (64 * rows);
            const int64_t n = std::max<int64_t>(1, std::min(classes / 8, std::max(512 / along, std::min<int64_t>(512, by_traffic))));
            p->grad_each = (classes + n - 1) / n;
            p->grad_groups = (int)((classes + p->grad_each - 1) / p->grad_each);
            p->Np = up_to(rows, 4);
        }
        auto grads = [&](auto& g, int64_t m, int64_t K) {
            g.deal = deal_of(m, features, K);
            g.m = dealt_tiles(m, g.deal); g.along = dealt_tiles(features, g.deal);
            const int64_t step = mpcnn::kDirectK * g.deal, all = (int64_t)g.m * g.along;   // (a step of each wave)
            const int64_t most = std::max<int64_t>(1, std::min<int64_t>(32, K / (4 * step)));
            const int64_t n = std::min(most, std::max<int64_t>(1, 4 * kCUs / std::max<int64_t>(1, all)));
            g.each = (int)up_to(std::max<int64_t>(1, (K + n - 1) / n), step);
            g.splits = (int)std::max<int64_t>(1, (K + g.each - 1) / g.each);
        };
        grads(p->gx, rows, classes);
        grads(p->gw, classes, rows);
        p->stat_tiles = std::max<int64_t>(p->score_v, (classes + 127) / 128);   // (of the block product at most)
        p->stats = take(8 * p->stat_tiles * rows);
        p->label_score = take(4 * rows);
        p->lse = take(4 * p->Np);
        p->weight = take(4 * p->Np);
        p->loss_part = take(8 * (p->Np + 1));
        if (p->wide) p->x_split = take(x_split_bytes(rows, features));
        if (p->few) {
            p->score = take(4 * classes * p->Np);
            p->dx_part = take(4 * (int64_t)p->grad_groups * rows * features);
        } else if (train) {
            p->score = take(4 * classes * p->Np);
            p->dx_part = take(p->gx.splits > 1 ? 4 * p->gx.splits * rows * features : 0);
            p->dw_part = take(p->gw.splits > 1 ? 4 * p->gw.splits * classes * features : 0);
            p->db_part = take(4 * classes * ((rows + 63) / 64));
        }
        p->total = at;
        return true;
    }
    int64_t piece = std::min<int64_t>(classes, kMaxPiece);
    auto bound = [&](int64_t most) { if (piece > most) piece = std::max<int64_t>(256, most / 256 * 256); };
    bound(kMostResults / p->Np);
    p->most_piece = piece;
    bound(kWeightRoom / p->d_bytes);
    if (train) bound(kRoom / p->Np);
    p->piece = piece;
    const int64_t pieces = (classes + piece - 1) / piece;
    // (Np, not N, in what is planned from here on: the same for all rows of a block of 64, as most_bytes wants it)
    const int64_t N = p->N, Np = p->Np, D = p->D;
    // The scores' sums over the features are split, too, where their tiles leave compute units without work.  us, split and summed / whole, bf16 1000 x 4096
    // x 2000 36 / 44, 200 x 4000 x 3000 26 / 46, 100 x 4096 x 20000 46 / 54; fp32 2469 x 3084 x 776 69 / 75, 1000 x 2048 x 2000 45 / 54.
    p->sc = tiling_of(classes, Np, p->d_bytes / mpcnn::kBlockBytes, pieces == 1 ? 16 : 1, p->halves);
    p->stat_tiles = std::max((classes + 127) / 128 + pieces, (classes + mpcnn::kScoresSum - 1) / mpcnn::kScoresSum * (p->sc.splits > 1));
    p->score_part = take(p->sc.splits > 1 ? 4 * p->sc.splits * classes * N : 0);
    p->peaks = take(4 * 3 * mpcnn::kPeakGroups);
    p->stats = take(8 * p->stat_tiles * N);
    p->label_score = take(4 * N);
    p->lse = take(4 * N);
    p->weight = take(4 * N);
    p->loss_part = take(8 * (N + 1));
    p->x_rows = take(N * p->d_bytes);
    p->w_rows = take(piece * p->d_bytes);
    if (train) {
        p->dx = tiling_of(Np, D, p->v_blocks(piece), std::min<int64_t>(64, std::max<int64_t>(1, kPartRoom / (4 * Np * D))), p->halves);
        p->dw = tiling_of(piece, D, p->n_bytes / mpcnn::kBlockBytes, std::min<int64_t>(64, std::max<int64_t>(1, kPartRoom / (4 * piece * D))), p->halves);
        p->x_cols = take(D * p->n_bytes);
        if (p->keep) p->score = take(classes * p->Np * 4);
        p->delta = take(piece * p->n_bytes);
        p->db_part = take(p->Np / 64 * piece * 4);
        if (p->dx_parts()) p->dx_part = take(4 * (int64_t)p->dx.splits * N * D);
        if (p->dw.splits > 1) p->dw_part = take(4 * (int64_t)p->dw.splits * piece * D);
    }
    p->total = at;
    return true;
}

// What is enough for every call with at most so many rows.  The sizes of a plan do not only grow with the rows: at 17 a way ends that leaves shares of the
// features' gradient, at the rows whose scores fill kRoom the scores are dropped (1000 features x 30011 classes, bf16: 35 MB for 16 rows, 10 MB for 17; 768 x 50257:
// 1.7 GB for 5106, 0.7 GB for 6207).  So every plan that may be the largest is made: up to 64 rows each; beyond, the choices are the same for all
// rows of a block of 32 (tiles of 32 rows, sums split in steps of 32, with little work) or of 64 (blocks and tiles, with much), and the sizes grow with the rows inside
// one, so each block's last is looked at, and the last rows of little work.  20-50 us for 8192 rows.
size_t most_bytes(int64_t rows, int64_t features, int64_t classes, int dtype, bool train)
{
    Plan p;
    size_t most = 0;
    auto look = [&](int64_t r) {
        if (make_plan(r, features, classes, dtype, train, &p)) most = std::max(most, p.total);
    };
    look(rows);
    if (!most) return 0;                                 // (bad sizes)
    for (int64_t r = 0; r < std::min<int64_t>(rows, 65); ++r) look(r);
    const int64_t little = (train ? kDirectWork : kDirectLossWork) / features / classes;
    if (little < rows) look(little);
    for (int64_t r = 96; r < rows; r = r < std::max(little, kWideRows) ? r + 32 : up_to(r + 1, 64)) look(r);
    return most;
}

// ---- launches of the product
template <int WM, int WN, int MT, int NT, bool HALVES, int RESULT, bool ACROSS>
mpcnn_status launch_instance(const mpcnn::ProductArgs& a, hipStream_t st)
{
    constexpr int lds = 2 * 32 * (WM * MT + WN * NT) * mpcnn::kBlockBytes;
    auto* kernel = &mpcnn::rows_product_kernel<WM, WN, MT, NT, HALVES, RESULT, ACROSS>;
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
    kernel<<<(unsigned)up_to(all, 8), 64 * WM * WN, lds, st>>>(a);
    return MPCNN_OK;
}
template <bool HALVES, int RESULT, bool ACROSS = false>
mpcnn_status launch_product(mpcnn::ProductArgs a, const Tiling& t, hipStream_t st)
{
    a.tiles_m = t.tiles_m; a.tiles_n = t.tiles_n; a.splits = t.splits; a.per_split = t.per_split;
    return t.big ? launch_instance<2, 4, 4, 2, HALVES, RESULT, ACROSS>(a, st) : launch_instance<2, 2, 2, 2, HALVES, RESULT, ACROSS>(a, st);
}

// Whether a product reads a matrix as it is: bf16, whole blocks at aligned addresses
template <typename T>
bool direct_operand(const void* m, int64_t pitch, int64_t features)
{
    return sizeof(T) == 2 && features % 64 == 0 && (uintptr_t)m % 16 == 0 && pitch % 8 == 0 && pitch * 512 < (1ll << 31);
}
// From so many class weights on the scores of little work are the block product's too, where it reads them as they are: 64 x 4096 x 32000 bf16
// 147 -> 68 us, 8 x 4096 x 128000 357 -> 197; 16 x 1024 x 32000 26 / 27
constexpr int64_t kBlockWeights = 40000000;

struct Call {
    const void *x, *w;
    int64_t x_pitch, w_pitch;
    const float* bias;
    const int32_t* labels;
    const float* roww;
    float *rowloss, *lse;
    double* loss;
    void* dx;
    int64_t dx_pitch;
    void* dw;
    float* db;
};

int join_groups_of(int N, int tiles)
{
    const int rows = mpcnn::join_rows(N, tiles);
    return (N + rows - 1) / rows;
}
void launch_join(const mpcnn::JoinArgs& j, hipStream_t st)
{
    const unsigned groups = (unsigned)join_groups_of(j.N, j.tiles);
    if (j.N <= mpcnn::kJoinLeast) mpcnn::rows_join_kernel<mpcnn::kJoinLeast, 1024><<<groups, 1024, 0, st>>>(j);
    else if (groups == 1) mpcnn::rows_join_kernel<mpcnn::kJoinMany, 1024><<<groups, 1024, 0, st>>>(j);
    else if (mpcnn::join_rows(j.N, j.tiles) == mpcnn::kJoinFew) mpcnn::rows_join_kernel<mpcnn::kJoinFew, 256><<<groups, 256, 0, st>>>(j);
    else mpcnn::rows_join_kernel<mpcnn::kJoinMany, 256><<<groups, 256, 0, st>>>(j);
}

mpcnn::FewArgs few_args(const Plan& p, const mpcnn::DirectArgs& a)
{
    mpcnn::FewArgs few{};
    few.x = a.x; few.w = a.w; few.x_pitch = a.x_pitch; few.w_pitch = a.w_pitch;
    few.N = a.N; few.D = a.D; few.V = p.V; few.score_row = a.score_row;
    few.bias = a.bias; few.mask = a.mask; few.scores = a.scores; few.stats = a.stats; few.stat_pitch = a.stat_pitch; few.label_score = a.label_score;
    return few;
}
// The scores of little work, or their statistics alone (a.scores null); notes how many tiles of classes these have, and of how many classes
template <typename T>
mpcnn_status direct_scores(const Plan& p, mpcnn::DirectArgs& a, char* x_split, int64_t* tile, hipStream_t st)
{
    const bool blocks = sizeof(T) == 2 && p.V * p.D >= kBlockWeights && direct_operand<T>(a.x, a.x_pitch, p.D) && direct_operand<T>(a.w, a.w_pitch, p.D);
    if (p.few_scores && !(blocks && p.N > 2)) {
        mpcnn::FewArgs few = few_args(p, a);
        few.each = *tile = p.score_each;
        mpcnn::launch_rows_few_scores<T>(few, (unsigned)p.score_v, st);
    } else if (blocks) {
        mpcnn::ProductArgs b{};
        b.A = (const char*)a.w; b.a_row = a.w_pitch * 2; b.B = (const char*)a.x; b.b_row = a.x_pitch * 2;
        b.M = a.V; b.N = p.N; b.blocks = p.D * 2 / mpcnn::kBlockBytes;
        b.bias = a.bias; b.labels = a.mask.labels; b.stats = a.stats; b.stat_pitch = a.stat_pitch; b.label_score = a.label_score; b.scores = a.scores; b.score_row = a.score_row;
        const Tiling t = tiling_of(p.V, p.N, b.blocks, 1, false);
        a.tiles = t.tiles_m;
        *tile = t.big ? 256 : 128;
        return launch_product<false, mpcnn::kScores>(b, t, st);
    } else if (sizeof(T) == 4 && p.wide) {
        *tile = 32;
        mpcnn::SplitArgs s{};
        s.x = (const float*)a.x; s.x_pitch = a.x_pitch; s.N = p.N; s.D = p.D; s.out = x_split;
        s.tiles = p.N <= 32 ? 1 : (int)(up_to(p.N, 64) / 32);
        const int64_t n = (int64_t)s.tiles * ((p.D + mpcnn::kDirectK - 1) / mpcnn::kDirectK) * 128;
        mpcnn::rows_split_kernel<<<(unsigned)std::min<int64_t>(4096, (n + 255) / 256), 256, 0, st>>>(s);
        a.x_split = s.out; a.x_tiles = s.tiles;
        if (s.tiles == 1) mpcnn::rows_wide_scores_kernel<1><<<(unsigned)p.score_v, 256, 0, st>>>(a);
        else mpcnn::rows_wide_scores_kernel<2><<<(unsigned)(p.score_v * (s.tiles / 2)), 256, 0, st>>>(a);
    } else {
        *tile = p.score_deal == 4 ? 32 : 64;
        const dim3 grid((unsigned)p.score_v, (unsigned)p.score_n);
        // rows of bf16 that begin between words (one row has no pitch)
        const bool odd = sizeof(T) == 2 && (((uintptr_t)a.x | (uintptr_t)a.w | 2 * (uint64_t)(p.N > 1 ? a.x_pitch : 0) | 2 * (uint64_t)(p.V > 1 ? a.w_pitch : 0)) & 2);
        if (odd) mpcnn::rows_direct_scores_kernel<T, sizeof(T) == 2><<<grid, 256, 0, st>>>(a);
        else mpcnn::rows_direct_scores_kernel<T, false><<<grid, 256, 0, st>>>(a);
    }
    return MPCNN_OK;
}

template <typename T>
mpcnn_status run_direct(const Plan& p, const Call& c, char* ws, hipStream_t st)
{
    mpcnn::DirectArgs a{};
    a.x = c.x; a.w = c.w; a.x_pitch = c.x_pitch; a.w_pitch = c.w_pitch;
    a.N = p.N; a.D = p.D; a.V = (int)p.V; a.bias = c.bias;
    a.mask = mpcnn::RowMask{c.labels, c.roww, (int)p.V};
    a.stats = (float2*)(ws + p.stats); a.label_score = (float*)(ws + p.label_score);
    a.score_row = p.Np; a.score_deal = p.score_deal; a.tiles = p.score_v;
    if (p.train) a.scores = (float*)(ws + p.score);
    int64_t tile = 0;
    const mpcnn_status rc = direct_scores<T>(p, a, p.wide ? ws + p.x_split : nullptr, &tile, st);
    if (rc != MPCNN_OK) return rc;
    // statistics joined with the derivative where there are few tiles of classes, by a launch of their own otherwise
    const bool joined = a.tiles > mpcnn::kDeltaFewTiles || p.few;
    a.lse = (float*)(ws + p.lse); a.weight = (float*)(ws + p.weight);
    double* const shares = (double*)(ws + p.loss_part);
    // (a workgroup takes several tiles of rows where that leaves four workgroups per compute unit: fewer sums over the rows to add up)
    constexpr int side = mpcnn::kDeltaSide;
    const int64_t v_tiles = p.train ? (p.V + side - 1) / side : 1, n_tiles = (p.N + side - 1) / side;
    a.batch = (int)std::max<int64_t>(1, std::min<int64_t>(n_tiles, v_tiles * n_tiles / (4 * kCUs)));
    const int along = (int)((n_tiles + a.batch - 1) / a.batch);
    int groups = along;
    if (joined) {
        mpcnn::JoinArgs j{};
        j.stats = a.stats; j.tiles = a.tiles; j.N = p.N; j.label_score = a.label_score; j.mask = a.mask;
        j.lse = a.lse; j.weight = a.weight; j.lse_out = c.lse; j.rowloss = c.rowloss;
        groups = join_groups_of(p.N, a.tiles);
        j.loss_part = groups == 1 && c.loss ? c.loss : shares;
        launch_join(j, st);
    } else {
        a.rowloss = c.rowloss; a.lse_out = c.lse;
        a.shares = groups == 1 && c.loss ? c.loss : shares;
    }
    a.loss = groups > 1 ? c.loss : nullptr; a.loss_part = shares; a.loss_parts = groups;
    if (p.few) {
        mpcnn::FewArgs few = few_args(p, a);
        few.lse = a.lse; few.weight = a.weight;
        few.dw = c.dw; few.db = c.db; few.each = p.grad_each;
        few.part = c.dx ? (float*)(ws + p.dx_part) : nullptr;
        const int each = mpcnn::few_columns(p.N);            // features of a thread
        few.columns = 16;
        while (few.columns < mpcnn::kFewThreads && each * few.columns < p.D) few.columns *= 2;
        if (c.dx || c.dw || c.db)
            mpcnn::launch_rows_few_grads<T>(few, dim3((unsigned)p.grad_groups, (unsigned)((p.D + each * few.columns - 1) / (each * few.columns))), st);
        few.parts = p.grad_groups; few.dx = c.dx; few.dx_pitch = c.dx_pitch;
        few.loss = a.loss; few.loss_part = a.loss_part; few.loss_parts = groups;
        if (few.part || few.loss)
            mpcnn::launch_rows_few_sum<T>(few, few.part ? (unsigned)(((int64_t)p.N * p.D + 63) / 64) : 1, st);
        HIP_TRY(hipGetLastError());
        return MPCNN_OK;
    }
    a.delta = p.train && (c.dx || c.dw || c.db);
    if (a.delta || !joined) {
        a.db = c.db;
        if (c.db && along > 1) { a.db_part = (float*)(ws + p.db_part); a.db_parts = along; }
        mpcnn::rows_direct_delta_kernel<<<dim3((unsigned)along, (unsigned)(a.delta ? v_tiles : 1)), 256, 0, st>>>(a);
    }
    if (p.train) {
        a.dx = c.dx; a.dx_pitch = c.dx_pitch; a.dw = c.dw;
        a.x_deal = p.gx.deal; a.w_deal = p.gw.deal; a.x_along = p.gx.along; a.w_along = p.gw.along;
        a.x_splits = p.gx.splits; a.x_each = p.gx.each; a.w_splits = p.gw.splits; a.w_each = p.gw.each;
        a.x_groups = c.dx ? p.gx.m * p.gx.along * p.gx.splits : 0;
        a.w_groups = c.dw ? p.gw.m * p.gw.along * p.gw.splits : 0;
        if (c.dx && p.gx.splits > 1) a.x_part = (float*)(ws + p.dx_part);
        if (c.dw && p.gw.splits > 1) a.w_part = (float*)(ws + p.dw_part);
    }
    a.db_groups = a.db_part ? (int)((p.V + 31) / 32) : 0;
    const int64_t all = (int64_t)a.x_groups + a.w_groups + a.db_groups;
    if (all || a.loss) mpcnn::rows_direct_grads_kernel<T><<<(unsigned)std::max<int64_t>(1, all), 256, 0, st>>>(a);
    if (a.x_part || a.w_part) {
        const int64_t n = (a.x_part ? (int64_t)p.N * p.D : 0) + (a.w_part ? p.V * p.D : 0);
        mpcnn::rows_direct_sum_kernel<T><<<(unsigned)std::min<int64_t>(8192, (n + 255) / 256), 256, 0, st>>>(a);
    }
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

template <typename T>
mpcnn_status run(const Plan& p, const Call& c, char* ws, hipStream_t st)
{
    constexpr bool H = sizeof(T) == 4;
    constexpr int kStore = H ? mpcnn::kStoreF32 : mpcnn::kStoreBf16;
    if (!p.N) {
        mpcnn::rows_none_kernel<<<(unsigned)std::min<int64_t>(4096, (p.V * p.D + 255) / 256), 256, 0, st>>>((char*)c.dw, p.V * p.D * (long)sizeof(T), c.db, p.V,
                                                                                                      c.loss);
        HIP_TRY(hipGetLastError());
        return MPCNN_OK;
    }
    if (p.direct) return run_direct<T>(p, c, ws, st);
    const mpcnn::RowMask every{}, mask{c.labels, c.roww, (int)p.V};
    unsigned* const x_peak = (unsigned*)(ws + p.peaks);
    unsigned *const w_peak = x_peak + mpcnn::kPeakGroups, *const wx_peak = c.roww ? w_peak + mpcnn::kPeakGroups : x_peak;   // wx: of the weighted features
    if constexpr (H) {
        mpcnn::PeakSet set{};
        int n = 0;
        auto peak = [&](const void* src, int64_t pitch, int64_t rows, const mpcnn::RowMask& m, int weighted, unsigned* words) {
            set.of[n++] = mpcnn::PeakArgs{(const float*)src, pitch, rows, p.D, m, weighted, words};
        };
        peak(c.x, c.x_pitch, p.N, mask, 0, x_peak);
        peak(c.w, c.w_pitch, p.V, every, 0, w_peak);
        if (p.train && c.roww) peak(c.x, c.x_pitch, p.N, mask, 1, wx_peak);
        mpcnn::rows_peak_kernel<<<dim3(mpcnn::kPeakGroups, (unsigned)n), 1024, 0, st>>>(set);
    }
    auto pack = [&](const void* src, int64_t pitch, int64_t R, char* rows, char* cols, int64_t col_bytes, const mpcnn::RowMask& m, const unsigned* words) {
        mpcnn::PackRowsArgs a{};
        a.src = src; a.pitch = pitch; a.R = (int)R; a.C = p.D;
        a.rows = rows; a.cols = cols; a.row_bytes = p.d_bytes; a.col_bytes = col_bytes;
        a.mask = m; a.peak = words; a.col_peak = wx_peak;
        const dim3 grid((unsigned)(H ? (R + 63) / 64 : (R + 127) / 128), (unsigned)((p.D + 63) / 64));
        (H ? mpcnn::rows_pack_kernel : mpcnn::rows_pack16_kernel)<<<grid, 256, 0, st>>>(a);
    };
    const bool x_direct = direct_operand<T>(c.x, c.x_pitch, p.D), w_direct = direct_operand<T>(c.w, c.w_pitch, p.D);
    if (!x_direct || p.train)
        pack(c.x, c.x_pitch, p.N, x_direct ? nullptr : ws + p.x_rows, p.train ? ws + p.x_cols : nullptr, p.n_bytes, mask, x_peak);

    // a piece's scores, or what becomes of them
    const int64_t piece = !p.train && w_direct ? p.most_piece : p.piece;
    const int d_blocks = (int)(p.d_bytes / mpcnn::kBlockBytes);
    int done = 0;                                        // tiles of classes
    auto scores = [&](int64_t v0, int64_t n_classes, const char* w_rows, int64_t w_row, mpcnn::ProductArgs a, bool delta) {
        a.A = w_rows; a.a_row = w_row;
        a.B = x_direct ? (const char*)c.x : ws + p.x_rows; a.b_row = x_direct ? c.x_pitch * 2 : p.d_bytes;
        a.M = (int)n_classes; a.N = p.N; a.blocks = d_blocks;
        a.a_peak = H ? w_peak : nullptr; a.b_peak = H ? x_peak : nullptr;
        a.bias = c.bias ? c.bias + v0 : nullptr;
        a.labels = c.labels; a.class0 = (int)v0;
        if (!delta && p.sc.splits > 1) {
            a.part = (float*)(ws + p.score_part);
            const mpcnn_status rc = launch_product<H, mpcnn::kPart>(a, p.sc, st);
            mpcnn::ScoresSumArgs s{};
            s.part = a.part; s.splits = p.sc.splits; s.M = a.M; s.N = a.N; s.a_peak = a.a_peak; s.b_peak = a.b_peak;
            s.bias = a.bias; s.labels = a.labels; s.stats = a.stats; s.label_score = a.label_score; s.scores = a.scores; s.score_row = a.score_row;
            done = (a.M + mpcnn::kScoresSum - 1) / mpcnn::kScoresSum;
            mpcnn::rows_scores_sum_kernel<H><<<dim3((unsigned)((a.N + 63) / 64), (unsigned)done), 256, 0, st>>>(s);
            return rc;
        }
        const Tiling t = tiling_of(n_classes, p.N, d_blocks, 1, H);
        if (!delta) done += t.tiles_m;
        return delta ? launch_product<H, mpcnn::kDelta>(a, t, st) : launch_product<H, mpcnn::kScores>(a, t, st);
    };
    // a piece's weights in blocks along the features, where they are not read as they are
    auto weights_of = [&](int64_t v0, int64_t n_classes) {
        if (!w_direct) pack((const char*)c.w + v0 * c.w_pitch * (int64_t)sizeof(T), c.w_pitch, n_classes, ws + p.w_rows, nullptr, 0, every, w_peak);
    };
    auto rows_at = [&](int64_t v0) { return w_direct ? (const char*)c.w + v0 * c.w_pitch * 2 : (const char*)(ws + p.w_rows); };
    const int64_t w_row = w_direct ? c.w_pitch * 2 : p.d_bytes;

    float* const score = p.keep ? (float*)(ws + p.score) : nullptr;
    const bool one_piece = p.V <= piece;                 // (its weights' blocks are there in the second round)
    for (int64_t v0 = 0; v0 < p.V; v0 += piece) {
        const int64_t n = std::min(piece, p.V - v0);
        weights_of(v0, n);
        mpcnn::ProductArgs a{};
        a.stats = (float2*)(ws + p.stats) + (int64_t)done * p.N; a.label_score = (float*)(ws + p.label_score);
        a.scores = p.keep ? score + v0 * p.Np : nullptr; a.score_row = p.Np;
        const mpcnn_status rc = scores(v0, n, rows_at(v0), w_row, a, false);
        if (rc != MPCNN_OK) return rc;
    }
    const int join_groups = join_groups_of(p.N, done);
    mpcnn::JoinArgs j{};
    j.stats = (const float2*)(ws + p.stats); j.tiles = done; j.N = p.N;
    j.label_score = (const float*)(ws + p.label_score); j.mask = mask;
    if (p.train) { j.lse = (float*)(ws + p.lse); j.weight = (float*)(ws + p.weight); }
    j.lse_out = c.lse; j.rowloss = c.rowloss;
    j.loss_part = c.loss ? (double*)(ws + p.loss_part) : nullptr;
    launch_join(j, st);

    mpcnn::FinishArgs fin{};
    fin.loss_part = j.loss_part; fin.loss_parts = join_groups; fin.loss = c.loss;
    if (!p.train) {
        if (c.loss) mpcnn::rows_finish_kernel<<<1, 256, 0, st>>>(fin);
        HIP_TRY(hipGetLastError());
        return MPCNN_OK;
    }
    for (int64_t v0 = 0; v0 < p.V; v0 += piece) {
        const int64_t n = std::min(piece, p.V - v0);
        const bool last = v0 + n == p.V;
        if (!one_piece && (!p.keep || c.dx)) weights_of(v0, n);
        char* const delta = c.dx || c.dw ? ws + p.delta : nullptr;
        float* const db_part = c.db ? (float*)(ws + p.db_part) : nullptr;
        if (p.keep) {
            mpcnn::DeltaArgs d{};
            d.scores = score + v0 * p.Np; d.score_row = p.Np; d.classes = (int)n; d.class0 = (int)v0; d.N = p.N;
            d.labels = c.labels; d.lse = j.lse; d.weight = j.weight;
            d.out = delta; d.out_bytes = p.n_bytes; d.db_part = db_part;
            mpcnn::rows_delta_kernel<H><<<dim3((unsigned)(p.Np / 64), (unsigned)((n + 63) / 64)), 256, 0, st>>>(d);
        } else {
            mpcnn::ProductArgs a{};
            a.lse = j.lse; a.weight = j.weight; a.delta = delta; a.delta_bytes = p.n_bytes; a.padded = (int)p.Np; a.db_part = db_part;
            const mpcnn_status rc = scores(v0, n, rows_at(v0), w_row, a, true);
            if (rc != MPCNN_OK) return rc;
        }
        fin.db_part = db_part; fin.tiles = (int)(p.Np / 64); fin.classes = n; fin.db = c.db ? c.db + v0 : nullptr;
        if (fin.db || fin.loss) mpcnn::rows_finish_kernel<<<fin.db ? (unsigned)((n + 31) / 32) : 1, 256, 0, st>>>(fin);
        fin.loss = nullptr;
        if (c.dx) {
            mpcnn::ProductArgs a{};
            a.A = ws + p.delta; a.a_row = p.n_bytes; a.a_bytes = n * p.n_bytes;
            a.B = rows_at(v0); a.b_row = w_row; a.b_bytes = (n - 1) * w_row + (w_direct ? 2 * (int64_t)p.D : p.d_bytes);
            a.M = p.N; a.N = p.D; a.blocks = (int)p.v_blocks(n);
            a.b_peak = H ? w_peak : nullptr;
            a.out = c.dx; a.out_row = c.dx_pitch; a.row_scale = j.weight; a.row_mask = !H;
            Tiling t = p.dx;
            t.per_split = (int)((a.blocks + t.splits - 1) / t.splits);
            mpcnn_status rc;
            if (p.dx_parts()) {
                a.part = (float*)(ws + p.dx_part); a.add = v0 > 0;
                rc = launch_product<H, mpcnn::kPart, true>(a, t, st);
                if (last) {
                    mpcnn::SumArgs sum{};
                    sum.part = a.part; sum.splits = t.splits; sum.M = p.N; sum.N = p.D; sum.out_row = c.dx_pitch;
                    sum.b_peak = a.b_peak; sum.halves = H; sum.row_scale = j.weight; sum.row_mask = !H; sum.out = c.dx; sum.out_bf16 = !H;
                    mpcnn::rows_sum_kernel<<<(unsigned)std::min<int64_t>(4096, ((int64_t)p.N * p.D + 255) / 256), 256, 0, st>>>(sum);
                }
            } else {
                rc = launch_product<H, kStore, true>(a, t, st);
            }
            if (rc != MPCNN_OK) return rc;
        }
        if (c.dw) {
            mpcnn::ProductArgs a{};
            a.A = ws + p.delta; a.a_row = p.n_bytes; a.B = ws + p.x_cols; a.b_row = p.n_bytes;
            a.M = (int)n; a.N = p.D; a.blocks = (int)(p.n_bytes / mpcnn::kBlockBytes);
            a.b_peak = H ? wx_peak : nullptr;
            a.out = (char*)c.dw + v0 * p.D * (int64_t)sizeof(T); a.out_row = p.D;
            Tiling t = p.dw;
            t.tiles_m = (int)((n + (t.big ? 255 : 127)) / (t.big ? 256 : 128));
            mpcnn_status rc;
            if (t.splits > 1) {
                a.part = (float*)(ws + p.dw_part);
                rc = launch_product<H, mpcnn::kPart>(a, t, st);
                mpcnn::SumArgs sum{};
                sum.part = a.part; sum.splits = t.splits; sum.M = n; sum.N = p.D; sum.out_row = p.D;
                sum.b_peak = a.b_peak; sum.halves = H; sum.out = a.out; sum.out_bf16 = !H;
                mpcnn::rows_sum_kernel<<<(unsigned)std::min<int64_t>(4096, (n * p.D + 255) / 256), 256, 0, st>>>(sum);
            } else {
                rc = launch_product<H, kStore>(a, t, st);
            }
            if (rc != MPCNN_OK) return rc;
        }
    }
    HIP_TRY(hipGetLastError());
    return MPCNN_OK;
}

mpcnn_status checked(int64_t rows, int64_t features, int64_t classes, mpcnn_dtype dtype, const Call& c, bool train, void* ws, size_t ws_bytes, void* stream)
{
    if (rows < 0 || features < 1 || classes < 1) return fail(MPCNN_EINVAL, "%lld rows, %lld features, %lld classes", (long long)rows, (long long)features, (long long)classes);
    if (dtype != MPCNN_F32 && dtype != MPCNN_BF16) return fail(MPCNN_EINVAL, "unknown type %d", (int)dtype);
    if (!c.w || !ws || (rows > 0 && (!c.x || !c.labels))) return fail(MPCNN_EINVAL, "null argument");
    if (c.x_pitch < features || c.w_pitch < features || (c.dx && c.dx_pitch < features))
        return fail(MPCNN_EINVAL, "a pitch is below the %lld features", (long long)features);
    const int64_t size = dtype == MPCNN_F32 ? 4 : 2, most_pitch = (int64_t)1 << 40;
    if (c.x_pitch > most_pitch || c.w_pitch > most_pitch || (c.dx && c.dx_pitch > most_pitch)) return fail(MPCNN_EINVAL, "a pitch is above 2^40");
    const uintptr_t typed = (uintptr_t)c.x | (uintptr_t)c.w | (uintptr_t)c.dx | (uintptr_t)c.dw;
    const uintptr_t words = (uintptr_t)c.bias | (uintptr_t)c.labels | (uintptr_t)c.roww | (uintptr_t)c.rowloss | (uintptr_t)c.lse | (uintptr_t)c.db;
    if (typed % size || words % 4 || (uintptr_t)c.loss % 8) return fail(MPCNN_EINVAL, "an address is no multiple of its element's size");
    Plan p;
    if (!make_plan(rows, features, classes, dtype, train, &p))
        return fail(MPCNN_EUNSUPPORTED, "%lld rows, %lld features, %lld classes: at most %lld, %lld, %lld", (long long)rows, (long long)features,
                    (long long)classes, (long long)kMaxRows, (long long)kMaxFeatures, (long long)kMaxClasses);
    if (ws_bytes < p.total) return fail(MPCNN_EWORKSPACE, "workspace %zu bytes, need %zu", ws_bytes, p.total);
    if ((uintptr_t)ws & 255u) return fail(MPCNN_EINVAL, "workspace must be 256-byte aligned");
    auto spread = [&](const void* m, int64_t n, int64_t pitch) { return Span{(uintptr_t)m, n ? (uint64_t)(((n - 1) * pitch + features) * size) : 0}; };
    const uint64_t n4 = 4 * (uint64_t)rows, v4 = 4 * (uint64_t)classes;
    const Span in[] = {spread(c.x, rows, c.x_pitch), spread(c.w, classes, c.w_pitch), {(uintptr_t)c.bias, v4}, {(uintptr_t)c.labels, n4}, {(uintptr_t)c.roww, n4}};
    const Span out[] = {{(uintptr_t)ws, p.total}, {(uintptr_t)c.rowloss, n4}, {(uintptr_t)c.lse, n4}, {(uintptr_t)c.loss, 8},
                        spread(c.dx, rows, c.dx_pitch), spread(c.dw, classes, features), {(uintptr_t)c.db, v4}};
    for (size_t i = 0; i < sizeof out / sizeof *out; ++i) {
        for (const Span& s : in)
            if (meet(out[i], s)) return fail(MPCNN_EINVAL, "an output or the workspace overlaps an input");
        for (size_t j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return fail(MPCNN_EINVAL, "two outputs, or one and the workspace, overlap");
    }
    return dtype == MPCNN_F32 ? run<float>(p, c, (char*)ws, (hipStream_t)stream) : run<mpcnn::bf16>(p, c, (char*)ws, (hipStream_t)stream);
}

// Classes whose scores can be kept: workgroups of 32 classes and 64 rows (128 at most) in one launch along them
constexpr int64_t kMostKept = (int64_t)1 << 27;
static_assert(kMostKept / 32 * 2 < kMostGroups && kMaxRows / 32 <= kMostSide, "a launch has them");

// What class_scores needs, and where: each grows with the rows
struct ScoresRoom { int64_t row, tiles; size_t scores, stats, x_split, total; };
bool scores_room(const mpcnn::ClassScores& c, ScoresRoom* r)
{
    if (c.rows < 0 || c.rows > kMaxRows || c.features < 1 || c.features > kMaxFeatures || c.classes < 1 || c.classes > kMaxClasses) return false;
    if (c.classes > kMostKept) return false;
    size_t at = 0;
    auto take = [&](int64_t bytes) { const size_t o = at; at += (size_t)up_to(bytes, 256); return o; };
    r->row = up_to(c.rows, 4);
    r->scores = take(4 * c.classes * r->row);
    r->tiles = up_to((c.classes + 31) / 32, 8);
    r->stats = take(8 * r->tiles * c.rows);
    r->x_split = take(c.dtype == MPCNN_F32 ? x_split_bytes(std::min(c.rows, kWideRows), c.features) : 0);
    r->total = at + 256;                                       // (no rows: not nothing)
    return true;
}

}  // namespace

namespace mpcnn {

size_t class_scores_bytes(const ClassScores& c)
{
    ScoresRoom r;
    return scores_room(c, &r) ? r.total : 0;
}

mpcnn_status class_scores(const ClassScores& c, char* ws, KeptScores* kept, hipStream_t st)
{
    ScoresRoom r;
    if (!scores_room(c, &r)) return fail(MPCNN_EUNSUPPORTED, "%lld rows, %lld features, %lld classes", (long long)c.rows, (long long)c.features, (long long)c.classes);
    Plan p{};
    p.halves = c.dtype == MPCNN_F32; p.direct = true;
    p.N = (int)c.rows; p.D = (int)c.features; p.V = c.classes; p.Np = r.row;
    p.wide = wide_scores(p.halves, c.rows, c.features, c.classes);
    p.few_scores = few_scores(p.halves, c.rows, c.features, c.classes);
    plan_scores(&p, c.rows, c.features, c.classes);
    if (p.few_scores) {                    // (at most 256 classes a workgroup here: one tile)
        p.score_each = p.score_each > 128 ? 256 : p.score_each;
        p.score_v = (int)((c.classes + p.score_each - 1) / p.score_each);
    }
    DirectArgs a{};
    a.x = c.x; a.w = c.w; a.x_pitch = c.x_pitch; a.w_pitch = c.w_pitch;
    a.N = p.N; a.D = p.D; a.V = (int)p.V; a.bias = c.bias;
    a.stats = (float2*)(ws + r.stats); a.stat_pitch = r.tiles; a.scores = (float*)(ws + r.scores); a.score_row = r.row; a.score_deal = p.score_deal; a.tiles = p.score_v;
    int64_t tile = 0;
    const mpcnn_status rc = c.dtype == MPCNN_F32 ? direct_scores<float>(p, a, ws + r.x_split, &tile, st) : direct_scores<bf16>(p, a, nullptr, &tile, st);
    *kept = KeptScores{a.scores, r.row, a.stats, r.tiles, tile, a.tiles};
    return rc;
}

}  // namespace mpcnn

extern "C" {

size_t mpcnn_workspace_bytes_class(int64_t rows, int64_t features, int64_t classes, mpcnn_dtype dtype, int training)
{
    return dtype == MPCNN_F32 || dtype == MPCNN_BF16 ? most_bytes(rows, features, classes, dtype, training != 0) : 0;
}

size_t mpcnn_workspace_bytes_class_call(int64_t rows, int64_t features, int64_t classes, mpcnn_dtype dtype, int training)
{
    Plan p;
    if ((dtype != MPCNN_F32 && dtype != MPCNN_BF16) || !make_plan(rows, features, classes, dtype, training != 0, &p)) return 0;
    return p.total;
}

mpcnn_status mpcnn_class_loss(const void* x_dev, int64_t x_pitch, const void* w_dev, int64_t w_pitch, const float* bias_dev,
                              const int32_t* labels_dev, const float* roww_dev, int64_t rows, int64_t features, int64_t classes,
                              mpcnn_dtype dtype, float* rowloss_dev, float* lse_dev, double* loss_dev, void* ws_dev, size_t ws_bytes,
                              void* hip_stream)
{
    const Call c{x_dev, w_dev, x_pitch, w_pitch, bias_dev, labels_dev, roww_dev, rowloss_dev, lse_dev, loss_dev, nullptr, 0, nullptr, nullptr};
    return checked(rows, features, classes, dtype, c, false, ws_dev, ws_bytes, hip_stream);
}

mpcnn_status mpcnn_class_backward(const void* x_dev, int64_t x_pitch, const void* w_dev, int64_t w_pitch, const float* bias_dev,
                                  const int32_t* labels_dev, const float* roww_dev, int64_t rows, int64_t features, int64_t classes,
                                  mpcnn_dtype dtype, float* rowloss_dev, double* loss_dev, void* dx_dev, int64_t dx_pitch, void* dw_dev,
                                  float* db_dev, void* ws_dev, size_t ws_bytes, void* hip_stream)
{
    const Call c{x_dev, w_dev, x_pitch, w_pitch, bias_dev, labels_dev, roww_dev, rowloss_dev, nullptr, loss_dev, dx_dev, dx_pitch, dw_dev, db_dev};
    return checked(rows, features, classes, dtype, c, true, ws_dev, ws_bytes, hip_stream);
}

}  // extern "C"
