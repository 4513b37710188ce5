// Host side of the experts' products (include/flexmoe.h): argument checks, the
// choice of kernel and of the parts of the reduction, launches.
#include <algorithm>
#include <cmath>

#include "error.h"
#include "flexmoe.h"
#include "grouped.h"

using namespace flexmoe;

namespace {

constexpr long long kMaxStride = 1 << 21;  // elements: a tile's rows stay below 2^31 bytes apart
constexpr size_t kMostPartial = 256u << 20;  // bytes of partial sums that are worth joining
constexpr int kMaxInt8Depth = 131071;      // 128 * 128 * K stays below 2^31

bool misaligned(const void* p, uintptr_t mask) { return ((uintptr_t)p & mask) != 0; }

int elem_bytes(int dtype) { return dtype == FLEXMOE_BF16 ? 2 : 4; }

// D's strides with 0 replaced by the packed ones.
struct Strides {
    long long x, w, y, dw;
};

int check(const flexmoe_grouped_desc* D, bool int8, const char* who, Strides* st) {
    if (!D) return fail(FLEXMOE_EINVAL, "%s: desc is NULL", who);
    for (int dt : {D->dtype, D->dw_dtype})
        if (dt != FLEXMOE_F32 && dt != FLEXMOE_BF16)
            return fail(FLEXMOE_EDTYPE, "%s: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", who, dt);
    if (D->groups < 1 || D->groups > kMaxExperts)
        return fail(FLEXMOE_ESHAPE, "%s: groups = %d outside [1, %d]", who, D->groups, kMaxExperts);
    if (D->N < 1 || D->K < 1 || D->N > kMaxStride || D->K > kMaxStride)
        return fail(FLEXMOE_ESHAPE, "%s: N = %d, K = %d outside [1, 2^21]", who, D->N, D->K);
    if (int8 && D->K > kMaxInt8Depth) return fail(FLEXMOE_ESHAPE, "%s: K = %d above %d", who, D->K, kMaxInt8Depth);
    if (D->keep_axis < FLEXMOE_KEEP_NONE || D->keep_axis > FLEXMOE_KEEP_K)
        return fail(FLEXMOE_EINVAL, "%s: keep_axis = %d outside [0, 2]", who, D->keep_axis);
    if (D->max_rows < 0 || D->max_rows > (1 << 30)) return fail(FLEXMOE_ESHAPE, "%s: max_rows = %d outside [0, 2^30]", who, D->max_rows);
    const int ein = int8 ? 16 : 16 / elem_bytes(D->dtype), eout = 16 / elem_bytes(D->dtype), edw = 16 / elem_bytes(D->dw_dtype);
    *st = Strides{D->ldx ? D->ldx : D->K, D->ldw ? D->ldw : D->K, D->ldy ? D->ldy : D->N, D->lddw ? D->lddw : D->K};
    const struct { long long ld, least; int unit; const char* name; } all[] = {
        {st->x, D->K, ein, "ldx"}, {st->w, D->K, ein, "ldw"}, {st->y, D->N, eout, "ldy"}, {st->dw, D->K, edw, "lddw"}};
    for (const auto& s : all) {
        if (int8 && s.name[2] == 'd') continue;
        if (s.ld < s.least || s.ld > kMaxStride || s.ld % s.unit)
            return fail(FLEXMOE_ESHAPE, "%s: %s = %lld must be a multiple of %d in [%lld, 2^21]", who, s.name, s.ld, s.unit, s.least);
    }
    return FLEXMOE_OK;
}

int check_rows(const flexmoe_grouped_desc* D, int R, const char* who) {
    if (R < 0) return fail(FLEXMOE_EINVAL, "%s: R = %d is negative", who, R);
    if (R > D->max_rows) return fail(FLEXMOE_ESHAPE, "%s: R = %d above max_rows = %d", who, R, D->max_rows);
    return FLEXMOE_OK;
}

// Row tiles of `bm` rows over all groups at most: sum ceil(n_e / bm) <=
// ceil(R / bm) + E - 1, and every tile holds a row.
long long row_tiles_bound(int R, int E, int bm) { return std::min<long long>((long long)(R + bm - 1) / bm + E - 1, R); }

// How a product is cut into workgroups.
enum Tiles { kMid = 0, kSlim = 1, kBig = 2, kFew = 3 };
struct Plan {
    GroupedForm form;
    GroupedElem elem;
    Tiles tiles;
    int splits;
    size_t workspace;
};

constexpr int kUnits = 256;  // compute units

// About the microseconds of a product on one kind of tiles with the reduction in
// `splits` parts, from what the host knows (not how rows and widths spread).
// Fitted to 3500 timings of 260 drawn products (1 to 128 groups, 1 to 32768
// rows, sides of 24 to 20480, every form and type, 1 to 13 parts).  On 515 other
// draws its choice takes 5 % more time on average than the fastest of those
// tried, at most 16 % more in 9 of 10, 1.85 times at worst.  It misses most where
// memory bounds a last round that is not full: 60 groups of 1408 x 2048 without
// widths, bf16, 1024 rows 89 us on 128-row tiles (32-row ones: 62), 4096 rows 100 on
// 256-row tiles (128-row ones: 84).
//   tiles     a K tile of 128 bytes costs a 256 x 256 tile 0.5 + 0.16 us per 64
//             rows; a 128 x 128 tile alone on its compute unit 0.17 + 0.14 us
//             per 32 rows (fp32: 0.1 + 0.45), two that share it 1.7 times that
//             (fp32: 2.1); n of up to four 32 x 128 tiles that share it n times
//             0.1 + 0.08 us per 16 rows (fp32: 0.1 + 0.15), at least 0.45; a tile
//             3.3, 1 or 1.5 us beside that; a last round of tiles that is not
//             full costs 0.7 of the missing part
//   memory    every operand and C once at 6.5 TB/s (32 x 128 tiles, but fp32: 5.7), 6 us at
//             least
//   together  the longer of the two and a quarter of the other
//   joining   a launch, and the parts written and read
// A width keeps 0.6 of what it limits.
double product_us(const flexmoe_grouped_desc& D, GroupedForm form, GroupedElem elem, Tiles kind, int splits, int R) {
    const int side = kind == kBig ? kGroupBigTile : kGroupTile, rows_of = kind == kFew ? kGroupFewRows : side;
    const int kd = elem == kElemI8 ? 128 : elem == kElemBf16 ? 64 : 32;
    const bool f32 = elem == kElemF32;
    const double es = 128.0 / kd, kept = D.keep_axis == FLEXMOE_KEEP_NONE ? 1.0 : 0.6;
    const int hit = std::max(1, std::min(D.groups, R));  // groups with rows, at most
    const int cols = form == kForward ? D.N : D.K;
    double row_tiles, tile_rows, depth, in, out;
    if (form == kWeightGrad) {
        row_tiles = (double)D.groups * ceil_div(D.N, rows_of);
        tile_rows = std::min(D.N, rows_of);
        depth = (D.groups > 1 ? 1.5 : 1.0) * R / D.groups;  // groups differ, and the longest is waited for
        in = (double)R * (D.N + (double)D.K) * es;
        out = (double)D.groups * D.N * cols;
    } else {
        const double rows = (double)R / hit;
        row_tiles = rows <= rows_of ? hit : R / (double)rows_of + 0.5 * hit;
        tile_rows = std::min<double>(rows, rows_of);
        depth = form == kForward ? D.K : D.N;
        in = (double)hit * D.N * D.K * es * kept + R * depth * es;
        out = (double)R * cols;
    }
    const double out_bytes = out * ((form == kWeightGrad ? D.dw_dtype : D.dtype) == FLEXMOE_BF16 ? 2 : 4);
    const double per_unit = row_tiles * ceil_div(cols, side) * splits / kUnits;
    const double k = std::ceil(std::ceil(depth / kd) / splits);
    auto rounds = [](double w) {
        w = std::max(1.0, w);
        return w + 0.7 * (std::ceil(w) - w);
    };
    double tiles_us;
    if (kind == kBig) {
        tiles_us = 3.5 + rounds(per_unit) * (3.3 + k * kept * (0.5 + 0.16 * std::ceil(tile_rows / 64)));
    } else if (kind == kFew) {
        const double step = 0.1 + (f32 ? 0.15 : 0.08) * std::ceil(tile_rows / 16);
        const double shared = std::min(std::max(per_unit, 1.0), 4.0) * step;
        tiles_us = 3.5 + rounds(per_unit / 4) * (1.5 + k * (per_unit > 1 ? kept : 1.0) * std::max(0.45, shared));
    } else {
        const double step = f32 ? 0.1 + 0.45 * std::ceil(tile_rows / 32) : 0.17 + 0.14 * std::ceil(tile_rows / 32);
        tiles_us = per_unit <= 1 ? 4.5 + k * step : 3.5 + rounds(per_unit / 2) * (1.0 + k * kept * step * (f32 ? 2.1 : 1.7));
    }
    const double memory_us = 6.0 + (in + out_bytes) / (kind == kFew && !f32 ? 5.7e6 : 6.5e6);
    double us = std::max(tiles_us, memory_us) + 0.25 * std::min(tiles_us, memory_us);
    if (splits > 1) us += 3.0 + 2 * splits * out * 4 / 5.6e6;
    return us;
}

// The plan of a call whose workspace holds `room` bytes of partial sums.
Plan plan(const flexmoe_grouped_desc& D, GroupedForm form, bool int8, int R, size_t room) {
    Plan pl{form, int8 ? kElemI8 : D.dtype == FLEXMOE_BF16 ? kElemBf16 : kElemF32, kMid, 1, 0};
    const long long cols = form == kForward ? D.N : D.K;
    const long long out = (form == kWeightGrad ? (long long)D.groups * D.N : (long long)R) * ((cols + 3) / 4 * 4) * 4;
    double best = 1e30;
    for (Tiles kind : {kMid, kFew, kBig}) {
        if ((kind == kBig && pl.elem == kElemF32) || (kind == kFew && form == kWeightGrad)) continue;
        for (int splits = 1; splits <= 64; splits = splits < 4 ? splits + 1 : splits * 3 / 2) {
            // parts of at least one K tile
            const int kd = pl.elem == kElemI8 ? 128 : pl.elem == kElemBf16 ? 64 : 32;
            const double depth = form == kWeightGrad ? (double)R / D.groups : form == kForward ? D.K : D.N;
            if (splits > 1 && (depth < (double)kd * splits || (size_t)(out * splits) > room)) break;
            const double us = product_us(D, form, pl.elem, kind, splits, R);
            if (us < best) {
                best = us;
                pl.tiles = kind;
                pl.splits = splits;
            }
        }
    }
    // A weight gradient that is not split is bound by its stores while groups
    // are short: four small workgroups per compute unit, whose stores and
    // requests cover each other.  Against 256 x 256 tiles, 60 groups of 1408 x
    // 2048 at 68 / 136 / 273 / 546 rows each: 140 to 181, 176 to 212, 226 to 258,
    // 317 to 344 us; 8 of 14336 x 4096 at 512 / 1024 / 2048: 769 to 739, 1156 to
    // 1096, 2177 to 1823.
    // (fp32 only up to 1024 rows: those workgroups have no registers for a second
    // level of sums.)
    if (form == kWeightGrad && pl.splits == 1 && R < 512LL * D.groups && (pl.elem == kElemBf16 || R <= 1024)) pl.tiles = kSlim;
    if (pl.splits > 1) pl.workspace = (size_t)(out * pl.splits);
    return pl;
}

int launch(const flexmoe_grouped_desc* D, const Strides& st, GroupedForm form, bool int8, int R, const void* a, const void* b, void* c,
           const float* sa, const float* sb, const int32_t* offsets, const int32_t* keep, int accumulate, void* ws, size_t ws_bytes,
           hipStream_t s, const char* who) {
    int rc = check_rows(D, R, who);
    if (rc) return rc;
    if (R == 0 && form != kWeightGrad) return FLEXMOE_OK;
    if ((R > 0 && (!a || !b)) || !c || !offsets) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    if ((D->keep_axis != FLEXMOE_KEEP_NONE) != (keep != nullptr))
        return fail(FLEXMOE_EINVAL, "%s: keep goes with keep_axis (%d)", who, D->keep_axis);
    if (misaligned(a, 15) || misaligned(b, 15) || misaligned(c, 15)) return fail(FLEXMOE_EINVAL, "%s: matrices must be 16-byte aligned", who);
    if (misaligned(offsets, 3) || misaligned(keep, 3) || misaligned(sa, 3) || misaligned(sb, 3))
        return fail(FLEXMOE_EINVAL, "%s: offsets, keep and scales must be 4-byte aligned", who);
    if (!ws) ws_bytes = 0;
    if (misaligned(ws, 255)) return fail(FLEXMOE_EWORKSPACE, "%s: workspace must be 256-byte aligned", who);
    const Plan pl = plan(*D, form, int8, R, std::min(ws_bytes, kMostPartial));
    GroupedParams p{};
    p.a = a, p.b = b, p.c = c, p.sa = sa, p.sb = sb, p.offsets = offsets, p.keep = keep, p.partial = ws;
    p.E = D->groups, p.R = R, p.N = D->N, p.K = D->K, p.keep_axis = D->keep_axis;
    p.slim = pl.tiles == kSlim;
    // Weights of 96 MB and more are not found in the 256 MB last-level cache by
    // the next call of a model's next layer (weights of several layers in turn:
    // 134 MB 32.5 -> 28.1 us, 346 MB 65.0 -> 57.8, 1.2 GB 120 -> 108 with the hint;
    // 67 MB 14.7 -> 18.7, 73 MB 17.8 -> 20.9).
    p.once = form != kWeightGrad && (double)D->groups * D->N * D->K * (int8 ? 1 : elem_bytes(D->dtype)) >= 96e6;
    p.splits = pl.splits, p.accumulate = accumulate;
    p.out_bf16 = (form == kWeightGrad ? D->dw_dtype : D->dtype) == FLEXMOE_BF16;
    if (form == kForward) p.lda = st.x, p.ldb = st.w, p.ldc = st.y;
    else if (form == kInputGrad) p.lda = st.y, p.ldb = st.w, p.ldc = st.x;
    else p.lda = st.y, p.ldb = st.x, p.ldc = st.dw;
    const int cols = form == kForward ? D->N : D->K;
    const int side = pl.tiles == kBig ? kGroupBigTile : kGroupTile;
    p.tiles_c = ceil_div(cols, side);
    p.tiles_r = ceil_div(D->N, side);
    const long long row_tiles = form == kWeightGrad ? (long long)D->groups * p.tiles_r
                                                    : row_tiles_bound(R, D->groups, pl.tiles == kFew ? kGroupFewRows : side);
    const long long tiles = row_tiles * p.tiles_c * p.splits;
    if (tiles > (1LL << 23) - 64) return  // a launch's threads are fewer than 2^32
        fail(FLEXMOE_ESHAPE, "%s: %lld tiles are too many for one launch", who, tiles);
    hipError_t err = pl.tiles == kBig   ? launch_grouped_big(p, form, pl.elem, tiles, s)
                     : pl.tiles == kFew ? launch_grouped_few(p, form, pl.elem, tiles, s)
                                        : launch_grouped_mid(p, form, pl.elem, tiles, s);
    if (err == hipSuccess && p.splits > 1) err = launch_grouped_join(p, form, pl.elem, s);
    if (err != hipSuccess) return hip_fail(err, who);
    return FLEXMOE_OK;
}

size_t workspace_bytes(const flexmoe_grouped_desc* D, int R, bool int8, const char* who) {
    Strides st;
    if (check(D, int8, who, &st) || check_rows(D, R, who)) return 0;
    size_t most = 256;  // 0 stands for an error
    // Fewer rows may use more: their reductions are split further.  Not every
    // smaller R is looked at; one between takes what there is.
    for (int form = kForward; form <= (int8 ? kForward : kWeightGrad); ++form)
        for (int r = R; r > 0; r = r > 64 ? r * 15 / 16 : r - 1)
            most = std::max(most, plan(*D, (GroupedForm)form, int8, r, kMostPartial).workspace);
    return (most + 255) & ~size_t(255);
}

}  // namespace

extern "C" {

size_t flexmoe_grouped_workspace_bytes(const flexmoe_grouped_desc* desc, int32_t R) {
    return workspace_bytes(desc, R, false, "grouped_workspace_bytes");
}

int flexmoe_grouped_forward(const flexmoe_grouped_desc* desc, int32_t R, const void* x, const void* w, const int32_t* offsets,
                            const int32_t* keep, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    Strides st;
    const int rc = check(desc, false, "grouped_forward", &st);
    return rc ? rc
              : launch(desc, st, kForward, false, R, x, w, y, nullptr, nullptr, offsets, keep, 0, workspace, workspace_bytes,
                       (hipStream_t)stream, "grouped_forward");
}

int flexmoe_grouped_input_grad(const flexmoe_grouped_desc* desc, int32_t R, const void* dy, const void* w, const int32_t* offsets,
                               const int32_t* keep, void* dx, void* workspace, size_t workspace_bytes, void* stream) {
    Strides st;
    const int rc = check(desc, false, "grouped_input_grad", &st);
    return rc ? rc
              : launch(desc, st, kInputGrad, false, R, dy, w, dx, nullptr, nullptr, offsets, keep, 0, workspace, workspace_bytes,
                       (hipStream_t)stream, "grouped_input_grad");
}

int flexmoe_grouped_weight_grad(const flexmoe_grouped_desc* desc, int32_t R, const void* dy, const void* x, const int32_t* offsets,
                                const int32_t* keep, void* dw, int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    Strides st;
    const int rc = check(desc, false, "grouped_weight_grad", &st);
    if (rc) return rc;
    if (accumulate != 0 && accumulate != 1) return fail(FLEXMOE_EINVAL, "grouped_weight_grad: accumulate = %d must be 0 or 1", accumulate);
    return launch(desc, st, kWeightGrad, false, R, dy, x, dw, nullptr, nullptr, offsets, keep, accumulate, workspace, workspace_bytes,
                  (hipStream_t)stream, "grouped_weight_grad");
}

int flexmoe_quantize_rows(int32_t rows, int32_t cols, int32_t dtype, const void* x, const void* x_gate, int64_t ldx, void* q, int64_t ldq,
                          float* scale, void* stream) {
    const char* who = "quantize_rows";
    if (dtype != FLEXMOE_F32 && dtype != FLEXMOE_BF16)
        return fail(FLEXMOE_EDTYPE, "%s: dtype %d is neither FLEXMOE_F32 nor FLEXMOE_BF16", who, dtype);
    if (rows < 0) return fail(FLEXMOE_EINVAL, "%s: rows = %d is negative", who, rows);
    if (cols < 1 || cols > kMaxStride) return fail(FLEXMOE_ESHAPE, "%s: cols = %d outside [1, 2^21]", who, cols);
    const int unit = 16 / elem_bytes(dtype);
    if (!ldx) ldx = cols;
    if (!ldq) ldq = cols;
    if (ldx < cols || ldx > kMaxStride || ldx % unit)
        return fail(FLEXMOE_ESHAPE, "%s: ldx = %lld must be a multiple of %d in [%d, 2^21]", who, (long long)ldx, unit, cols);
    if (ldq < cols || ldq > kMaxStride || ldq % 16)
        return fail(FLEXMOE_ESHAPE, "%s: ldq = %lld must be a multiple of 16 in [%d, 2^21]", who, (long long)ldq, cols);
    if (rows == 0) return FLEXMOE_OK;
    if (!x || !q || !scale) return fail(FLEXMOE_EINVAL, "%s: a pointer is NULL", who);
    if (misaligned(x, 15) || misaligned(x_gate, 15) || misaligned(q, 15) || misaligned(scale, 3))
        return fail(FLEXMOE_EINVAL, "%s: matrices must be 16-byte aligned, scales 4-byte", who);
    const hipError_t err = x_gate ? launch_quantize_rows(x_gate, x, (size_t)ldx, (int8_t*)q, (size_t)ldq, scale, rows, cols,
                                                         dtype == FLEXMOE_BF16, (hipStream_t)stream)
                                  : launch_quantize_rows(x, nullptr, (size_t)ldx, (int8_t*)q, (size_t)ldq, scale, rows, cols,
                                                         dtype == FLEXMOE_BF16, (hipStream_t)stream);
    if (err != hipSuccess) return hip_fail(err, who);
    return FLEXMOE_OK;
}

size_t flexmoe_quantized_workspace_bytes(const flexmoe_grouped_desc* desc, int32_t R) {
    return workspace_bytes(desc, R, true, "quantized_workspace_bytes");
}

int flexmoe_quantized_forward(const flexmoe_grouped_desc* desc, int32_t R, const void* q, const float* q_scale, const void* w,
                         const float* w_scale, const int32_t* offsets, const int32_t* keep, void* y, void* workspace,
                         size_t workspace_bytes, void* stream) {
    Strides st;
    const int rc = check(desc, true, "quantized_forward", &st);
    if (rc) return rc;
    if (R > 0 && (!q_scale || !w_scale)) return fail(FLEXMOE_EINVAL, "quantized_forward: a scale pointer is NULL");
    return launch(desc, st, kForward, true, R, q, w, y, q_scale, w_scale, offsets, keep, 0, workspace, workspace_bytes, (hipStream_t)stream,
                  "quantized_forward");
}

}  // extern "C"
