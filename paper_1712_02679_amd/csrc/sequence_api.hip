// sequence_api.hip -- the C ABI of adacomp_sequence.h: argument checks and launch sequences.
#include <cmath>
#include <cstddef>

#include "layers_checks.h"
#include "sequence_plan.h"

namespace adacomp {

constexpr uint64_t kMost = uint64_t(1) << 31, kMostVocab = uint64_t(1) << 30, kMostCols = uint64_t(1) << 20, kMostValues = uint64_t(1) << 38;

static bool embed_sizes(uint64_t rows, uint64_t vocab, uint64_t cols)
{
    return rows < kMost && vocab != 0 && vocab <= kMostVocab && cols <= kMostCols && rows * cols <= kMostValues;
}

static int embed_args(const adacomp_embed_t *op, const adacomp_dropout_t *dropout, EmbedArgs &a)
{
    a = EmbedArgs();
    if (!op || op->dtype > ADACOMP_DTYPE_F16 || op->reserved != 0) return ADACOMP_EINVAL;
    if (!embed_sizes(op->rows, op->vocab, op->cols)) return ADACOMP_EINVAL;
    if (op->index_bytes != 4 && op->index_bytes != 8) return ADACOMP_EINVAL;
    if (int rc = drop_args(dropout, a.drop)) return rc;
    if (op->rows != 0 && op->cols != 0 && !op->tokens) return ADACOMP_EINVAL;
    if (!aligned(op->tokens, op->index_bytes)) return ADACOMP_EALIGN;
    a.tokens = op->tokens;
    a.stride = op->stride;
    a.rows = uint32_t(op->rows);
    a.vocab = op->vocab;
    a.cols = op->cols;
    a.groups = (op->cols + 7u) / 8u;
    a.index64 = op->index_bytes == 8;
    a.scale = op->scale;
    return ADACOMP_OK;
}

static int steps_args(const adacomp_steps_t *steps, const adacomp_recurrence_t *op, bool written, StepsArgs &out)
{
    out = StepsArgs();
    if (!steps) return ADACOMP_EINVAL;
    if (!steps->data && op->batch != 0 && op->length != 0 && op->channels != 0) return ADACOMP_EINVAL;
    if (!aligned(steps->data, element_bytes(op->dtype))) return ADACOMP_EALIGN;
    if (written) {   // rows that are written lie apart
        const auto apart = [op](uint32_t count, int64_t stride) { return count < 2u || stride >= int64_t(op->channels) || stride <= -int64_t(op->channels); };
        if (!apart(op->batch, steps->batch_stride) || !apart(op->length, steps->row_stride)) return ADACOMP_EINVAL;
    }
    out = {steps->data, steps->batch_stride, steps->row_stride};
    return ADACOMP_OK;
}

// Whether 64 rows lie within 32 bits of the first one.
static bool near_rows(const StepsArgs &s) { return s.row >= 0 && s.row < int64_t(1) << 23; }

// Whether a result shares no memory with what is read, as far as the tensors' first and last bytes say.
static bool apart(const StepsArgs &out, const StepsArgs &in, const adacomp_recurrence_t *op)
{
    const auto ends = [op](const StepsArgs &s, int64_t &low, int64_t &high) {
        const int64_t e = int64_t(element_bytes(op->dtype)), batch = (int64_t(op->batch) - 1) * s.batch, rows = (int64_t(op->length) - 1) * s.row;
        low = int64_t(reinterpret_cast<uintptr_t>(s.data)) + (std::min<int64_t>(batch, 0) + std::min<int64_t>(rows, 0)) * e;
        high = int64_t(reinterpret_cast<uintptr_t>(s.data)) + (std::max<int64_t>(batch, 0) + std::max<int64_t>(rows, 0) + op->channels) * e;
    };
    if (!out.data || !in.data) return true;
    int64_t low, high, in_low, in_high;
    ends(out, low, high);
    ends(in, in_low, in_high);
    return high <= in_low || in_high <= low;
}

// The same of two [batch, channels] states, either of which may be NULL.
static bool states_apart(const float *one, const float *other, const adacomp_recurrence_t *op)
{
    const uint64_t bytes = uint64_t(op->batch) * op->channels * 4u, a = reinterpret_cast<uintptr_t>(one), b = reinterpret_cast<uintptr_t>(other);
    return !one || !other || a + bytes <= b || b + bytes <= a;
}

static bool recurrence_sizes(uint64_t batch, uint64_t length, uint64_t channels)
{
    return batch < kMost && length < kMost && channels <= kMostCols && batch * length < kMost;
}

static int recurrence_args(const adacomp_recurrence_t *op, RecurrenceArgs &a)
{
    a = RecurrenceArgs();
    if (!op || op->dtype > ADACOMP_DTYPE_F16 || !recurrence_sizes(op->batch, op->length, op->channels)) return ADACOMP_EINVAL;
    if (!aligned(op->bias, 4) || !aligned(op->lengths, 4)) return ADACOMP_EALIGN;
    a.bias = op->bias;
    a.lengths = op->lengths;
    a.resets = op->resets;
    a.resets_stride = op->resets_stride;
    a.batch = op->batch;
    a.length = op->length;
    a.channels = op->channels;
    a.slabs = (op->channels + kSlab - 1u) / kSlab;
    a.kept = (op->length + ADACOMP_RECURRENCE_KEEP - 1u) / ADACOMP_RECURRENCE_KEEP;
    const RecurrenceForm form = recurrence_form(op->batch, op->length, op->channels);
    a.segments = form.segments;
    a.segment = form.segment;
    return ADACOMP_OK;
}

// Bytes of the sums of the bias gradient; changes of the parts follow them.
static size_t recurrence_sums(const RecurrenceForm &form, uint64_t batch, uint64_t channels) { return pad256(size_t(batch) * form.segments * channels * 4u); }

static bool finite_at_least(float x, float least) { return std::isfinite(x) && x >= least; }

static int distill_args(const adacomp_distill_t *op, const void *logits, const float *dloss, const void *dlogits, DistillArgs &a)
{
    a = DistillArgs();
    if (!op || op->dtype > ADACOMP_DTYPE_F16 || op->rows >= kMost || op->vocab == 0 || op->vocab > kMostVocab) return ADACOMP_EINVAL;
    if (op->top > ADACOMP_TEACHER_TOP_MAX) return ADACOMP_EINVAL;
    const float per = 1.f / op->temperature;
    if (!(op->temperature > 0.f) || !std::isfinite(op->temperature) || !std::isfinite(per) || per == 0.f) return ADACOMP_EINVAL;
    if (!finite_at_least(op->soft, 0.f) || !finite_at_least(op->hard, 0.f) || !std::isfinite(op->scale)) return ADACOMP_EINVAL;
    const float soft_loss = op->soft * op->temperature * op->temperature, soft_grad = op->soft * op->temperature;
    if (!std::isfinite(soft_loss)) return ADACOMP_EINVAL;
    const size_t e = element_bytes(op->dtype);
    if (op->top != 0) {
        if (op->teacher_dtype > ADACOMP_DTYPE_F16 || (op->tokens_bytes != 4 && op->tokens_bytes != 8)) return ADACOMP_EINVAL;
        if (op->rows != 0 && (!op->teacher_tokens || !op->teacher_logits)) return ADACOMP_EINVAL;
        if (!aligned(op->teacher_tokens, op->tokens_bytes) || !aligned(op->teacher_logits, element_bytes(op->teacher_dtype))) return ADACOMP_EALIGN;
    }
    if (op->targets) {
        if (op->targets_bytes != 4 && op->targets_bytes != 8) return ADACOMP_EINVAL;
        if (!aligned(op->targets, op->targets_bytes)) return ADACOMP_EALIGN;
    }
    if (op->rows != 0 && !logits) return ADACOMP_EINVAL;
    if (dlogits && op->rows > 1 && op->dlogits_stride < op->vocab) return ADACOMP_EINVAL;
    if (!aligned(logits, e) || !aligned(dlogits, e) || !aligned(dloss, 4)) return ADACOMP_EALIGN;
    const bool taught = op->top != 0 && op->soft > 0.f, told = op->targets && op->hard > 0.f;
    a.logits = logits;
    a.dlogits = const_cast<void *>(dlogits);
    a.teacher_tokens = op->teacher_tokens;
    a.teacher_logits = op->teacher_logits;
    a.targets = told ? op->targets : nullptr;
    a.dloss = dloss;
    a.logits_stride = op->logits_stride;
    a.dlogits_stride = op->dlogits_stride;
    a.tokens_stride = op->tokens_stride;
    a.teacher_stride = op->teacher_stride;
    a.rows = op->rows;
    a.vocab = op->vocab;
    a.top = taught ? op->top : 0u;
    a.tokens64 = op->tokens_bytes == 8;
    a.targets64 = op->targets_bytes == 8;
    a.teacher_dtype = op->teacher_dtype;
    a.per_temperature = per;
    a.hard = op->hard;
    a.soft_loss = soft_loss;
    a.soft_grad = soft_grad;
    a.scale = op->scale;
    return ADACOMP_OK;
}

}  // namespace adacomp

using namespace adacomp;

extern "C" {

int adacomp_embed_forward(const adacomp_embed_t *op, const float *table, void *y, const adacomp_dropout_t *dropout, void *hip_stream)
{
    EmbedArgs a;
    if (int rc = embed_args(op, dropout, a)) return rc;
    if (a.rows == 0 || a.cols == 0) return ADACOMP_OK;
    if (!table || !y || (a.rows > 1 && a.stride < a.cols)) return ADACOMP_EINVAL;
    if (!aligned(table, 4) || !aligned(y, element_bytes(op->dtype))) return ADACOMP_EALIGN;
    a.table = table;
    a.rows_of = y;
    return launch_embed_forward(a, op->dtype, hip_stream);
}

size_t adacomp_embed_workspace_bytes(uint64_t rows, uint32_t vocab, uint32_t cols)
{
    if (!embed_sizes(rows, vocab, cols)) return 0;
    const EmbedForm f = embed_form(uint32_t(rows), vocab, cols);
    return pad256((size_t(vocab) + 1u) * 4u) + pad256(size_t(rows) * sizeof(EmbedPlace)) + pad256(size_t(f.pieces) * 2u * f.pitch * 4u);
}

int adacomp_embed_backward(const adacomp_embed_t *op, const void *dy, float *dtable, const adacomp_dropout_t *dropout, int accumulate,
                           void *workspace, size_t workspace_bytes, void *hip_stream)
{
    EmbedArgs a;
    if (int rc = embed_args(op, dropout, a)) return rc;
    if (a.cols == 0) return ADACOMP_OK;
    if (!dtable || (a.rows != 0 && !dy)) return ADACOMP_EINVAL;
    if (!aligned(dtable, 4) || !aligned(dy, element_bytes(op->dtype))) return ADACOMP_EALIGN;
    if (int rc = workspace_check(workspace, workspace_bytes, adacomp_embed_workspace_bytes(op->rows, op->vocab, op->cols))) return rc;
    a.rows_of = const_cast<void *>(dy);
    a.dtable = dtable;
    a.accumulate = accumulate != 0;
    a.first = static_cast<uint32_t *>(workspace);
    char *behind = static_cast<char *>(workspace) + pad256((size_t(a.vocab) + 1u) * 4u);
    a.order = reinterpret_cast<EmbedPlace *>(behind);
    a.parts = reinterpret_cast<float *>(behind + pad256(size_t(a.rows) * sizeof(EmbedPlace)));
    return launch_embed_backward(a, op->dtype, hip_stream);
}

size_t adacomp_recurrence_workspace_bytes(uint32_t batch, uint32_t length, uint32_t channels)
{
    if (!recurrence_sizes(batch, length, channels)) return 0;
    const RecurrenceForm form = recurrence_form(batch, length, channels);
    const size_t sums = recurrence_sums(form, batch, channels);
    return std::max<size_t>(256u, sums + (form.segments > 1u ? 2u * sums : 0u));
}

int adacomp_recurrence_forward(const adacomp_recurrence_t *op, const adacomp_steps_t *x, const adacomp_steps_t *forget, const adacomp_steps_t *out,
                               const float *first, const adacomp_steps_t *y, float *last, float *states, void *workspace, size_t workspace_bytes,
                               void *hip_stream)
{
    RecurrenceArgs a;
    if (int rc = recurrence_args(op, a)) return rc;
    if (int rc = steps_args(x, op, false, a.x)) return rc;
    if (int rc = steps_args(forget, op, false, a.forget)) return rc;
    if (out)
        if (int rc = steps_args(out, op, false, a.out)) return rc;
    if (int rc = steps_args(y, op, true, a.y)) return rc;
    if (!aligned(first, 4) || !aligned(last, 4) || !aligned(states, 4)) return ADACOMP_EALIGN;
    if (a.batch == 0 || a.channels == 0) return ADACOMP_OK;
    if (int rc = workspace_check(workspace, workspace_bytes, adacomp_recurrence_workspace_bytes(op->batch, op->length, op->channels))) return rc;
    a.first = first;
    a.last = last;
    a.states = states;
    a.near_rows = near_rows(a.x) && near_rows(a.forget) && near_rows(a.out) && near_rows(a.y);
    a.apart = states_apart(first, last, op) && apart(a.y, a.x, op) && apart(a.y, a.forget, op) && apart(a.y, a.out, op);
    a.changes = reinterpret_cast<float *>(static_cast<char *>(workspace) + recurrence_sums({a.segments, a.segment}, a.batch, a.channels));
    return launch_recurrence_forward(a, op->dtype, hip_stream);
}

int adacomp_recurrence_backward(const adacomp_recurrence_t *op, const adacomp_steps_t *dy, const adacomp_steps_t *x, const adacomp_steps_t *forget,
                                const adacomp_steps_t *out, const float *states, const float *dlast, const adacomp_steps_t *dx,
                                const adacomp_steps_t *dforget, const adacomp_steps_t *dout, float *dbias, float *dfirst, int accumulate,
                                void *workspace, size_t workspace_bytes, void *hip_stream)
{
    RecurrenceArgs a;
    if (int rc = recurrence_args(op, a)) return rc;
    if (!out != !dout) return ADACOMP_EINVAL;
    if (int rc = steps_args(dy, op, false, a.y)) return rc;
    if (int rc = steps_args(x, op, false, a.x)) return rc;
    if (int rc = steps_args(forget, op, false, a.forget)) return rc;
    if (int rc = steps_args(dx, op, true, a.dx)) return rc;
    if (int rc = steps_args(dforget, op, true, a.dforget)) return rc;
    if (out) {
        if (int rc = steps_args(out, op, false, a.out)) return rc;
        if (int rc = steps_args(dout, op, true, a.dout)) return rc;
    }
    if (!aligned(states, 4) || !aligned(dlast, 4) || !aligned(dfirst, 4) || !aligned(dbias, 4)) return ADACOMP_EALIGN;
    if (a.channels == 0) return ADACOMP_OK;
    if (a.batch != 0) {
        if (a.length != 0 && !states) return ADACOMP_EINVAL;
        if (int rc = workspace_check(workspace, workspace_bytes, adacomp_recurrence_workspace_bytes(op->batch, op->length, op->channels))) return rc;
        a.near_rows = near_rows(a.x) && near_rows(a.forget) && near_rows(a.out) && near_rows(a.y) && near_rows(a.dx) && near_rows(a.dforget) && near_rows(a.dout);
        a.apart = states_apart(dlast, dfirst, op);
        for (const StepsArgs *out : {&a.dx, &a.dforget, &a.dout})
            for (const StepsArgs *in : {&a.x, &a.forget, &a.out, &a.y}) a.apart = a.apart && apart(*out, *in, op);
        a.first = dlast;
        a.last = dfirst;
        a.states = const_cast<float *>(states);
        a.dbias_parts = dbias ? static_cast<float *>(workspace) : nullptr;
        a.changes = reinterpret_cast<float *>(static_cast<char *>(workspace) + recurrence_sums({a.segments, a.segment}, a.batch, a.channels));
        if (int rc = launch_recurrence_backward(a, op->dtype, hip_stream)) return rc;
    }
    if (!dbias) return ADACOMP_OK;
    return launch_bias_sum({a.dbias_parts, dbias, a.batch * a.segments, a.channels, accumulate != 0}, hip_stream);
}

int adacomp_distill_forward(const adacomp_distill_t *op, const void *logits, float *loss, float *lse, const float *dloss, void *dlogits,
                            void *hip_stream)
{
    DistillArgs a;
    if (int rc = distill_args(op, logits, dloss, dlogits, a)) return rc;
    if (!aligned(loss, 4) || !aligned(lse, 4)) return ADACOMP_EALIGN;
    if (a.rows == 0) return ADACOMP_OK;
    if (!loss) return ADACOMP_EINVAL;
    a.loss = loss;
    a.lse = lse;
    return launch_distill(a, op->dtype, dlogits ? LOSS_GRAD : LOSS, hip_stream);
}

int adacomp_distill_backward(const adacomp_distill_t *op, const void *logits, const float *lse, const float *dloss, void *dlogits,
                             void *hip_stream)
{
    DistillArgs a;
    if (int rc = distill_args(op, logits, dloss, dlogits, a)) return rc;
    if (!aligned(lse, 4)) return ADACOMP_EALIGN;
    if (a.rows == 0) return ADACOMP_OK;
    if (!lse || !dlogits) return ADACOMP_EINVAL;
    a.lse = const_cast<float *>(lse);
    return launch_distill(a, op->dtype, GRAD, hip_stream);
}

}  // extern "C"
