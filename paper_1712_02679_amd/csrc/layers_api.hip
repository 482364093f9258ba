// layers_api.hip -- the C ABI of adacomp_layers.h: argument checks and launch sequences.
#include <cmath>
#include <cstddef>

#include "layers_plan.h"

namespace adacomp {

static size_t element_bytes(uint32_t dtype) { return dtype == ADACOMP_DTYPE_F32 ? 4u : 2u; }
static bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
static size_t pad256(size_t x) { return (x + 255u) & ~size_t(255); }

static int drop_args(const adacomp_dropout_t *drop, DropArgs &out)
{
    out = DropArgs();
    if (!drop) return ADACOMP_OK;
    if (!(drop->p >= 0.f && drop->p < 1.f) || drop->reserved != 0) return ADACOMP_EINVAL;
    const double threshold = std::floor(double(drop->p) * 65536.0 + 0.5);
    if (threshold >= 65536.0) return ADACOMP_EINVAL;
    if (!aligned(drop->step, 8)) return ADACOMP_EALIGN;
    out.step = drop->step;
    out.seed_lo = uint32_t(drop->seed);
    out.seed_hi = uint32_t(drop->seed >> 32);
    out.stream_lo = uint32_t(drop->stream);
    out.stream_hi = uint32_t(drop->stream >> 32);
    out.threshold = uint32_t(threshold);
    out.on = out.threshold != 0;
    out.factor = float(65536.0 / (65536.0 - threshold));
    return ADACOMP_OK;
}

static int view_args(const adacomp_view_t *view, const adacomp_bias_softmax_t *op, size_t element, bool written, ViewArgs &out)
{
    out = ViewArgs();
    if (!view) return ADACOMP_EINVAL;
    const bool empty = op->batch == 0 || op->heads == 0 || op->queries == 0 || op->keys == 0;
    if (!view->data && !empty) return ADACOMP_EINVAL;
    if (!aligned(view->data, element)) return ADACOMP_EALIGN;
    if (written) {   // rows that are written lie apart
        const auto apart = [op](uint32_t count, int64_t stride) { return count < 2u || stride >= int64_t(op->keys) || stride <= -int64_t(op->keys); };
        if (!apart(op->batch, view->batch_stride) || !apart(op->heads, view->head_stride) || !apart(op->queries, view->row_stride)) return ADACOMP_EINVAL;
    }
    out = {view->data, view->batch_stride, view->head_stride, view->row_stride};
    return ADACOMP_OK;
}

static bool softmax_sizes(uint64_t batch, uint64_t heads, uint64_t queries, uint64_t keys, uint64_t distance)
{
    const uint64_t most = uint64_t(1) << 31;
    if (batch >= most || heads > (uint64_t(1) << 20) || queries >= most || keys >= (uint64_t(1) << 30)) return false;
    if (distance == 0 || distance > ADACOMP_BIAS_DISTANCE_MAX) return false;
    if (batch * heads >= most) return false;
    return batch * heads * queries < most;
}

// Parts of the workspace of the softmax calls, in bytes.
struct SoftmaxRoom {
    size_t stats, sums;
    size_t all() const { return stats + sums; }
};

static SoftmaxRoom softmax_room(const SoftmaxArgs &a, const SoftmaxForm &form, bool backward)
{
    SoftmaxRoom room = {0, 0};
    if (form.parts > 1u) room.stats = pad256(size_t(a.batch) * a.heads * a.queries * form.parts * 8u);
    if (backward && a.heads) room.sums = pad256(size_t(a.heads) * softmax_back_groups_most(uint64_t(a.batch) * a.queries, a.heads, form) * a.places * 4u);
    return room;
}

// The distances key - query that a call can have, as far as the host knows, in the map's numbering.
static void softmax_places(SoftmaxArgs &a)
{
    const int64_t far = a.distance, ends = 2 * far;
    int64_t low = 0, high = ends;
    if (!a.query_starts) {
        low = std::min(std::max(far - (int64_t(a.query_start) + a.queries - 1), int64_t(0)), ends);
        high = std::min(std::max(far + int64_t(a.keys) - 1 - a.query_start, low), ends);
    }
    if (a.causal) high = std::min(high, far);   // no key behind its query
    low = std::min(low, high);
    a.first_place = uint32_t(low);
    a.places = uint32_t(high - low + 1);
}

// What the two softmax calls check alike.
static int softmax_args(const adacomp_bias_softmax_t *op, const adacomp_view_t *scores, const adacomp_dropout_t *dropout, SoftmaxArgs &a)
{
    a = SoftmaxArgs();
    if (!op || op->dtype > ADACOMP_DTYPE_F16) return ADACOMP_EINVAL;
    if (!softmax_sizes(op->batch, op->heads, op->queries, op->keys, op->max_distance)) return ADACOMP_EINVAL;
    if (op->n_buckets == 0 || op->n_buckets > 2u * ADACOMP_BIAS_DISTANCE_MAX + 1u || !op->table || !op->map) return ADACOMP_EINVAL;
    if (!aligned(op->table, 4) || !aligned(op->map, 4) || !aligned(op->query_starts, 4) || !aligned(op->key_lengths, 4)) return ADACOMP_EALIGN;
    if (int rc = view_args(scores, op, element_bytes(op->dtype), false, a.scores)) return rc;
    if (op->mask.data)
        if (int rc = view_args(&op->mask, op, 1, false, a.mask)) return rc;
    if (int rc = drop_args(dropout, a.drop)) return rc;
    a.query_starts = op->query_starts;
    a.key_lengths = op->key_lengths;
    a.map = op->map;
    a.table = op->table;
    a.batch = op->batch;
    a.heads = op->heads;
    a.queries = op->queries;
    a.keys = op->keys;
    a.causal = op->causal != 0;
    a.n_buckets = op->n_buckets;
    a.distance = op->max_distance;
    a.query_start = op->query_start;
    a.scale = op->scale;
    softmax_places(a);
    return ADACOMP_OK;
}

static int workspace_check(const void *workspace, size_t bytes, size_t needed)
{
    if (needed == 0) return ADACOMP_OK;
    if (!workspace) return ADACOMP_EINVAL;
    if (!aligned(workspace, 16)) return ADACOMP_EALIGN;
    return bytes < needed ? ADACOMP_EWORKSPACE : ADACOMP_OK;
}

}  // namespace adacomp

using namespace adacomp;

extern "C" {

int adacomp_dropout(const void *x, const void *residual, void *y, uint64_t rows, uint64_t cols, uint64_t x_stride,
                    uint64_t residual_stride, uint64_t y_stride, uint32_t dtype, const adacomp_dropout_t *dropout, void *hip_stream)
{
    const uint64_t most = uint64_t(1) << 31;
    if (dtype > ADACOMP_DTYPE_F16 || !dropout || rows >= most || cols >= most) return ADACOMP_EINVAL;
    DropoutLaunch a = {};
    if (int rc = drop_args(dropout, a.drop)) return rc;
    if (rows == 0 || cols == 0) return ADACOMP_OK;
    if (!x || !y || (rows > 1 && y_stride < cols)) return ADACOMP_EINVAL;
    const size_t e = element_bytes(dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(residual, e)) return ADACOMP_EALIGN;
    a.x = x; a.residual = residual; a.y = y;
    a.x_stride = x_stride; a.residual_stride = residual_stride; a.y_stride = y_stride;
    a.cols = uint32_t(cols); a.groups = uint32_t((cols + 7u) / 8u);
    a.dtype = dtype;
    const uint64_t step = std::max<uint64_t>(1, (uint64_t(1) << 30) / a.groups);   // groups of a launch are counted in 32 bits
    for (uint64_t first = 0; first < rows; first += step) {
        a.first_row = first;
        a.rows = uint32_t(std::min(step, rows - first));
        if (int rc = launch_dropout(a, hip_stream)) return rc;
    }
    return ADACOMP_OK;
}

static int norm_check(const adacomp_norm_t *norm)
{
    if (!norm || norm->dtype > ADACOMP_DTYPE_F16 || norm->rows >= (uint64_t(1) << 31)) return ADACOMP_EINVAL;
    return norm->cols == 0 || norm->cols > ADACOMP_NORM_COLS_MAX ? ADACOMP_EINVAL : ADACOMP_OK;
}

int adacomp_norm_forward(const adacomp_norm_t *norm, const void *x, const void *residual, const float *gamma, const float *beta,
                         float eps, const adacomp_dropout_t *dropout, void *z, void *y, float *mean, float *rstd, void *hip_stream)
{
    if (int rc = norm_check(norm)) return rc;
    if (!(eps >= 0.f)) return ADACOMP_EINVAL;
    NormForward a = {};
    if (int rc = drop_args(dropout, a.drop)) return rc;
    if (norm->rows == 0) return ADACOMP_OK;
    const bool rows_apart = norm->rows == 1 || (norm->y_stride >= norm->cols && (!z || norm->z_stride >= norm->cols));
    if (!x || !y || y == z || !rows_apart) return ADACOMP_EINVAL;
    const size_t e = element_bytes(norm->dtype);
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(z, e) || !aligned(y, e)) return ADACOMP_EALIGN;
    if (!aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return ADACOMP_EALIGN;
    a.x = x; a.residual = residual; a.gamma = gamma; a.beta = beta;
    a.z = z; a.y = y; a.mean = mean; a.rstd = rstd;
    a.x_stride = norm->x_stride; a.residual_stride = norm->residual_stride;
    a.z_stride = norm->z_stride; a.y_stride = norm->y_stride;
    a.all_rows = norm->rows; a.cols = norm->cols; a.eps = eps;
    return launch_norm_forward(a, norm->dtype, hip_stream);
}

size_t adacomp_norm_workspace_bytes(uint64_t rows, uint64_t cols)
{
    if (rows >= (uint64_t(1) << 31) || cols == 0 || cols > ADACOMP_NORM_COLS_MAX) return 0;
    return pad256(std::max<size_t>(size_t(norm_parts(rows, uint32_t(cols))) * 2u * norm_pitch(uint32_t(cols)) * 4u, 16u));
}

int adacomp_norm_backward(const adacomp_norm_t *norm, const void *dy, const void *dz_add, const void *z, const float *mean,
                          const float *rstd, const float *gamma, const adacomp_dropout_t *dropout, void *dz, void *dx, float *dgamma,
                          float *dbeta, int accumulate, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = norm_check(norm)) return rc;
    NormBackward a = {};
    if (int rc = drop_args(dropout, a.drop)) return rc;
    if ((dx && !dropout) || (dx && dx == dz)) return ADACOMP_EINVAL;
    if (!aligned(gamma, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4)) return ADACOMP_EALIGN;
    const bool sums = dgamma || dbeta;
    const uint32_t parts = norm_parts(norm->rows, norm->cols);
    if (norm->rows != 0) {
        if (!dy || !z || !mean || !rstd || !dz) return ADACOMP_EINVAL;
        if (norm->rows > 1 && (norm->dz_stride < norm->cols || (dx && norm->dx_stride < norm->cols))) return ADACOMP_EINVAL;
        const size_t e = element_bytes(norm->dtype);
        if (!aligned(dy, e) || !aligned(dz_add, e) || !aligned(z, e) || !aligned(dz, e) || !aligned(dx, e)) return ADACOMP_EALIGN;
        const uint32_t pitch = norm_pitch(norm->cols);
        if (sums)
            if (int rc = workspace_check(workspace, workspace_bytes, size_t(parts) * 2u * pitch * 4u)) return rc;
        a.dy = dy; a.dz_add = dz_add; a.z = z; a.mean = mean; a.rstd = rstd; a.gamma = gamma;
        a.dz = dz; a.dx = dx;
        a.partial = sums ? static_cast<float *>(workspace) : nullptr;
        a.dy_stride = norm->dy_stride; a.dz_add_stride = norm->dz_add_stride; a.z_stride = norm->z_stride;
        a.dz_stride = norm->dz_stride; a.dx_stride = norm->dx_stride;
        a.rows = uint32_t(norm->rows); a.cols = norm->cols; a.pitch = pitch;
        if (int rc = launch_norm_backward(a, norm->dtype, parts, hip_stream)) return rc;
    }
    if (!sums) return ADACOMP_OK;
    const NormReduce r = {static_cast<const float *>(workspace), dgamma, dbeta, parts, norm_pitch(norm->cols), norm->cols, accumulate != 0};
    return launch_norm_reduce(r, hip_stream);
}

int adacomp_relative_buckets(uint32_t n_buckets, uint32_t max_distance, int both_directions, int32_t *map)
{
    if (!map || max_distance == 0 || max_distance > ADACOMP_BIAS_DISTANCE_MAX) return ADACOMP_EINVAL;
    if (n_buckets > 2u * ADACOMP_BIAS_DISTANCE_MAX + 1u || (both_directions && n_buckets % 2u)) return ADACOMP_EINVAL;
    const uint32_t count = both_directions ? n_buckets / 2u : n_buckets, single = count / 2u;
    if (count < 2u || max_distance <= single) return ADACOMP_EINVAL;
    for (int64_t d = -int64_t(max_distance); d <= int64_t(max_distance); ++d) {
        uint32_t first = 0, n = d < 0 ? uint32_t(-d) : 0u;
        if (both_directions && d > 0) { first = count; n = uint32_t(d); }
        if (n >= single) {
            const double part = std::log(double(n) / single) / std::log(double(max_distance) / single);
            n = std::min(count - 1u, single + uint32_t(part * (count - single) + 1e-9));
        }
        map[d + max_distance] = int32_t(first + n);
    }
    return ADACOMP_OK;
}

size_t adacomp_bias_softmax_workspace_bytes(uint32_t batch, uint32_t heads, uint32_t queries, uint32_t keys, uint32_t max_distance)
{
    if (!softmax_sizes(batch, heads, queries, keys, max_distance)) return 0;
    // in whatever form a call goes: parts of rows as the keys make them, sums of every distance for as many workgroups as there can be
    const uint32_t parts = softmax_form(keys, 1, false).parts;
    const size_t rows_of_head = size_t(batch) * queries * parts, rows = rows_of_head * heads;
    const size_t groups = heads ? std::min<size_t>(rows_of_head, std::max(1u, kMostResident * kComputeUnits / heads)) : 0u;
    return std::max<size_t>(256u, (parts > 1u ? pad256(rows * 8u) : 0u) + pad256(groups * heads * (2u * max_distance + 1u) * 4u));
}

int adacomp_bias_softmax_forward(const adacomp_bias_softmax_t *op, const adacomp_view_t *scores, const adacomp_view_t *probs, float *lse,
                                 const adacomp_dropout_t *dropout, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    SoftmaxArgs a;
    if (int rc = softmax_args(op, scores, dropout, a)) return rc;
    if (int rc = view_args(probs, op, element_bytes(op->dtype), true, a.out)) return rc;
    if (!aligned(lse, 4)) return ADACOMP_EALIGN;
    if (uint64_t(a.batch) * a.heads * a.queries == 0) return ADACOMP_OK;
    const SoftmaxForm form = softmax_form(a.keys, a.places, false);
    const SoftmaxRoom room = softmax_room(a, form, false);
    if (int rc = workspace_check(workspace, workspace_bytes, room.all())) return rc;
    a.lse = lse;
    a.part_stats = static_cast<float *>(workspace);
    return launch_softmax_forward(a, op->dtype, form, hip_stream);
}

int adacomp_bias_softmax_backward(const adacomp_bias_softmax_t *op, const adacomp_view_t *scores, const float *lse,
                                  const adacomp_view_t *dprobs, const adacomp_dropout_t *dropout, const adacomp_view_t *dscores,
                                  float *dtable, int accumulate, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    SoftmaxArgs a;
    if (int rc = softmax_args(op, scores, dropout, a)) return rc;
    const size_t e = element_bytes(op->dtype);
    if (int rc = view_args(dprobs, op, e, false, a.in)) return rc;
    if (int rc = view_args(dscores, op, e, true, a.out)) return rc;
    if (!aligned(lse, 4) || !aligned(dtable, 4)) return ADACOMP_EALIGN;
    if (a.heads == 0) return ADACOMP_OK;
    const uint64_t rows_of_head = uint64_t(a.batch) * a.queries;
    const SoftmaxForm form = softmax_form(a.keys, a.places, true);
    SoftmaxRoom room = softmax_room(a, form, true);
    if (!dtable) room.sums = 0;
    char *base = static_cast<char *>(workspace);
    uint32_t groups = 0;
    if (rows_of_head != 0) {
        if (!lse) return ADACOMP_EINVAL;
        if (int rc = workspace_check(workspace, workspace_bytes, room.all())) return rc;
        a.lse = const_cast<float *>(lse);
        a.part_stats = reinterpret_cast<float *>(base);
        a.bias_sums = dtable ? reinterpret_cast<float *>(base + room.stats) : nullptr;
        if (int rc = launch_softmax_backward(a, op->dtype, form, groups, hip_stream)) return rc;
    }
    if (!dtable) return ADACOMP_OK;
    const BiasReduce r = {reinterpret_cast<const float *>(base + room.stats), a.map + a.first_place, dtable, a.heads, groups, a.places, a.n_buckets, accumulate != 0};
    return launch_bias_reduce(r, hip_stream);
}

}  // extern "C"
