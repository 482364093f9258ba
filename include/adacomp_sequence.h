/*
 * adacomp_sequence.h -- what a learner that works on tokens has besides matrix products and the calls of adacomp_layers.h: the
 * embedding that its step begins with, a gated linear recurrence, and the distillation loss that it ends with.
 *
 * The conventions are those of adacomp_layers.h: tensors of dtype with contiguous last dimensions, parameters (the embedding table,
 * the bias of the gates), their gradients, states, losses and the arithmetic in float32, results rounded once, sums in a fixed
 * order (a call repeats bit for bit), launches on hip_stream alone.  Token numbers are int32 or int64: index_bytes 4 or 8, aligned
 * to that.  A number outside 0 .. vocab - 1 stands for no token, wherever it is found.
 * Workspaces hold nothing between calls; calls that may run at the same time need one each.
 */
#ifndef ADACOMP_SEQUENCE_H
#define ADACOMP_SEQUENCE_H

#include "adacomp_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- embedding ------------------------------------------------------------------------------------ */

/* rows below 2^31; vocab 1 .. 2^30; cols up to 2^20; rows * cols up to 2^38; tokens [rows] contiguous; stride: of y or dy, in elements.
 * dropout may be NULL. */
typedef struct {
    uint64_t rows, stride;
    uint32_t vocab, cols, dtype, index_bytes;
    const void *tokens;
    float scale;
    uint32_t reserved; /* 0 */
} adacomp_embed_t;

/* y[r] = D(scale table[tokens[r]]), zeros where there is no token.  table [vocab, cols] float32. */
int adacomp_embed_forward(const adacomp_embed_t *op, const float *table, void *y, const adacomp_dropout_t *dropout, void *hip_stream);

/* Bytes of workspace of adacomp_embed_backward. */
size_t adacomp_embed_workspace_bytes(uint64_t rows, uint32_t vocab, uint32_t cols);

/* dtable[v] = sum over the rows r with token v of scale D(dy[r]), added up in the order of the rows in pieces that the sizes decide.
 * accumulate != 0 adds to what is there (rows of tokens that do not occur are left alone), 0 overwrites all of dtable.
 * Made for mini-batches: for each part of the vocabulary, of up to 512 tokens, the tokens of all rows are looked at, so that the time grows with
 * rows times vocab where both are large (64 columns bf16: 2^20 rows over 50000 tokens 0.57 ms, over 262144 1.05 ms). */
int adacomp_embed_backward(const adacomp_embed_t *op, const void *dy, float *dtable, const adacomp_dropout_t *dropout, int accumulate,
                           void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- gated linear recurrence ---------------------------------------------------------------------- */

/* Along each sequence, channel by channel, from the state h[-1] = first:
 *   a[t] = sigmoid(forget[t] + bias),  m[t] = a[t], or 0 where resets[t] != 0 (a document begins there: nothing of what was before it
 *   comes through, and no gradient goes back, NaN and infinities included)
 *   h[t] = m[t] h[t - 1] + (1 - a[t]) x[t],  y[t] = sigmoid(out[t]) h[t], or h[t] without out
 * Places from lengths[b] on are padding: not looked at, the state stays what it is, y and gradients are zeros there.
 * Backward, with G[t] = sigmoid(out[t]) dy[t] + m[t + 1] G[t + 1], at the sequence's last place dlast added:
 *   dx = (1 - a) G,  dforget = a (1 - a) (p - x) G with p[t] = h[t - 1], or 0 where resets[t] != 0,
 *   dout = sigmoid(out) sigmoid(-out) h dy,  dbias = sum of dforget over all places,  dfirst = m[0] G[0]
 * (an empty sequence: last = first, dfirst = dlast).
 *
 * The forward pass keeps the state before every ADACOMP_RECURRENCE_KEEP'th place, from which the backward pass makes the others
 * again: states [batch, ceil(length / ADACOMP_RECURRENCE_KEEP), channels].
 *
 * batch, length and their product below 2^31, channels up to 2^20.
 *   bias      [channels] or NULL: zeros
 *   lengths   device [batch], clamped to 0 .. length, or NULL: all of them
 *   resets    uint8 [batch, length] with the given stride, or NULL */
#define ADACOMP_RECURRENCE_KEEP 64u

typedef struct {
    const void *data;
    int64_t batch_stride, row_stride;
} adacomp_steps_t; /* [batch, length, channels] */

typedef struct {
    uint32_t batch, length, channels, dtype;
    const float *bias;
    const int32_t *lengths;
    const uint8_t *resets;
    int64_t resets_stride;
} adacomp_recurrence_t;

/* Bytes of workspace of the two calls below. */
size_t adacomp_recurrence_workspace_bytes(uint32_t batch, uint32_t length, uint32_t channels);

/* first, last  [batch, channels] float32, first NULL: zeros, last NULL: not wanted; they may be the same buffer
 * out          NULL: no gate
 * states       NULL: not wanted */
int adacomp_recurrence_forward(const adacomp_recurrence_t *op, const adacomp_steps_t *x, const adacomp_steps_t *forget, const adacomp_steps_t *out,
                               const float *first, const adacomp_steps_t *y, float *last, float *states, void *workspace, size_t workspace_bytes,
                               void *hip_stream);

/* out and dout are both given or both NULL.  dlast, dfirst [batch, channels] float32: dlast NULL: zeros, dfirst NULL: not wanted; they may be the same buffer;
 * dbias [channels] NULL: not wanted, accumulate != 0 adds to what is there, 0 overwrites. */
int adacomp_recurrence_backward(const adacomp_recurrence_t *op, const adacomp_steps_t *dy, const adacomp_steps_t *x, const adacomp_steps_t *forget,
                                const adacomp_steps_t *out, const float *states, const float *dlast, const adacomp_steps_t *dx,
                                const adacomp_steps_t *dforget, const adacomp_steps_t *dout, float *dbias, float *dfirst, int accumulate,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- distillation --------------------------------------------------------------------------------- */

#define ADACOMP_TEACHER_TOP_MAX 256u

/* The loss of each row of logits z, from what a teacher and a target say about it:
 *   p = softmax(t / temperature) over the teacher's top tokens (no tokens among them are left out, a token that stands there twice
 *       counts twice),  q = softmax(z / temperature),  lse = log(sum of exp(z / temperature)),  lse1 = log(sum of exp(z))
 *   loss = soft temperature^2 sum over the top tokens of p (log p - log q)  +  hard (lse1 - z[target])
 *   dlogits = scale dloss ( soft temperature (q - p)  +  hard (softmax(z) - [target]) )
 * A row has the first term if soft > 0 and one of its top tokens is a token with t above -infinity, the second if hard > 0 and its
 * target is a token.  A row with neither is padding: loss 0, gradient zeros, whatever it holds; gradient zeros too where dloss is 0.
 * -infinity in z, or in z / temperature as a float32, is a token that cannot be: q = 0.  A row of nothing else, and one with -infinity at
 * its target or at a top token with p > 0, has a loss of infinity; in the former all of q is 0.  A NaN or +infinity there makes the row NaN.
 * lse is a float32, and q of the backward pass as exact as that allows (off by 2^-24 of lse).
 * rows below 2^31; vocab 1 .. 2^30; top 0 .. ADACOMP_TEACHER_TOP_MAX, 0: no teacher; temperature > 0; soft, hard >= 0, finite.
 *   teacher_tokens, teacher_logits  [rows, top] with row strides; teacher_dtype is that of teacher_logits
 *   targets                         [rows] or NULL */
typedef struct {
    uint64_t rows;
    uint32_t vocab, dtype;
    uint64_t logits_stride, dlogits_stride;
    const void *teacher_tokens, *teacher_logits, *targets;
    uint64_t tokens_stride, teacher_stride;
    uint32_t top, teacher_dtype, tokens_bytes, targets_bytes;
    float temperature, soft, hard, scale;
} adacomp_distill_t;

/* loss [rows] float32.
 * lse [rows, 2] float32, for the backward pass: lse and lse1, 0 where the row has no such term; NULL: not wanted
 * dlogits NULL: not wanted; otherwise the gradient is computed in the same pass, dloss [rows] float32, NULL: ones */
int adacomp_distill_forward(const adacomp_distill_t *op, const void *logits, float *loss, float *lse, const float *dloss, void *dlogits,
                            void *hip_stream);

/* dlogits from the logits and the lse of the forward pass, with the same op (scale may differ).  It may be the logits' buffer. */
int adacomp_distill_backward(const adacomp_distill_t *op, const void *logits, const float *lse, const float *dloss, void *dlogits,
                             void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
