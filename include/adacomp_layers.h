/*
 * adacomp_layers.h -- the pieces between the matrix products of a learner's training step: dropout,
 * layer norm, and the masked softmax of attention scores with a learned relative position bias.
 *
 * Their learned parameters (gamma, beta, the bias table) are float32 layers of the learner's flat
 * weight buffer, and their gradients are written in float32 into the layers' places in the flat
 * gradient that adacomp_compress (adacomp.h) packs: summed over all rows in a fixed order, so that a
 * call repeats bit for bit.
 *
 * Conventions (those of adacomp.h, and)
 *   - dtype is the type of the tensors that have one value per row and column; parameters, their
 *     gradients, statistics and the arithmetic are float32.  A result is rounded once, to nearest even.
 *   - Every tensor's last dimension is contiguous; the other strides are in elements.  Addresses need
 *     the alignment of one element, parameters, statistics and index arrays that of 4 bytes, workspaces 16.
 *   - An output may be the same buffer as an input of the same strides; otherwise buffers must not overlap.
 *   - Calls only launch kernels on hip_stream: no allocation, no copy, no synchronisation; they can be
 *     captured in a graph.  The device is the one current in the calling thread.
 *   - A tensor without any element is no error: nothing is read, and gradients of parameters are zeros.
 */
#ifndef ADACOMP_LAYERS_H
#define ADACOMP_LAYERS_H

#include "adacomp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ADACOMP_DTYPE_F32 0u
#define ADACOMP_DTYPE_BF16 1u
#define ADACOMP_DTYPE_F16 2u

/* ---- dropout -------------------------------------------------------------------------------------- */

/* D(x): every value is kept with probability 1 - T / 65536, T = floor(p 65536 + 1/2), and then
 * multiplied by 65536 / (65536 - T), or replaced by zero.  Which values are kept is a function of
 * (seed, stream, row, column) alone: the mask is made again wherever it is needed, and the backward
 * pass is the same call on the gradient.
 *
 * The generator is Philox-4x32 with 7 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers:
 * as easy as 1, 2, 3", SC 2011): key = seed (low word first), counter = (column / 8, row, stream low word,
 * stream high word).  The four result words are eight 16-bit numbers, low half first, one for each of
 * 8 columns; a value is kept where its number is at least T.
 *   p      0 <= p < 1, and T below 65536
 *   stream what tells calls apart: a number per layer and training step
 *   step   NULL, or a device pointer to a number that is added to stream when the kernel runs, so that a
 *          captured graph draws another mask at every replay; 8-byte aligned */
typedef struct {
    float p;
    uint32_t reserved; /* 0 */
    uint64_t seed;
    uint64_t stream;
    const uint64_t *step;
} adacomp_dropout_t;

/* y = D(x), or with residual != NULL y = residual + D(x): tensors [rows, cols] with the given row strides.
 * rows and cols below 2^31. */
int adacomp_dropout(const void *x, const void *residual, void *y, uint64_t rows, uint64_t cols, uint64_t x_stride,
                    uint64_t residual_stride, uint64_t y_stride, uint32_t dtype, const adacomp_dropout_t *dropout,
                    void *hip_stream);

/* ---- layer norm ----------------------------------------------------------------------------------- */

#define ADACOMP_NORM_COLS_MAX 32768u

/* rows below 2^31, cols 1 .. ADACOMP_NORM_COLS_MAX; row strides of the call's tensors, in elements
 * (those of tensors that the call does not have are not looked at). */
typedef struct {
    uint64_t rows;
    uint32_t cols, dtype;
    uint64_t x_stride, residual_stride, z_stride, y_stride; /* forward */
    uint64_t dy_stride, dz_add_stride, dz_stride, dx_stride; /* backward, with z_stride */
} adacomp_norm_t;

/* z = x, D(x), residual + x or residual + D(x);  mean and var (divided by cols) of each row of z, from the
 * values before z is rounded;  rstd = 1 / sqrt(var + eps);  y = (z - mean) rstd gamma + beta.
 *   residual, dropout   may be NULL
 *   gamma, beta         [cols]; NULL: ones, zeros
 *   z                   where z goes, NULL if it is not wanted
 *   mean, rstd          [rows], NULL if they are not wanted
 * The backward pass needs z (x itself where there is neither residual nor dropout), mean and rstd.
 * eps >= 0. */
int adacomp_norm_forward(const adacomp_norm_t *norm, const void *x, const void *residual, const float *gamma,
                         const float *beta, float eps, const adacomp_dropout_t *dropout, void *z, void *y, float *mean,
                         float *rstd, void *hip_stream);

/* Bytes of workspace of adacomp_norm_backward.  Nothing in it is kept between calls. */
size_t adacomp_norm_workspace_bytes(uint64_t rows, uint64_t cols);

/* With h = (z - mean) rstd and g = dy gamma:
 *   dz = rstd (g - average(g) - h average(g h)) [+ dz_add], averages over the row: the gradient of z, and
 *        of the residual;  dz_add, may be NULL, is what arrives at z on other paths
 *   dx = D(dz), for dropout != NULL: the gradient of x;  dx may be NULL if it is not wanted, and must be
 *        without dropout, when it would be dz
 *   dgamma = sum over rows of dy h, dbeta = sum over rows of dy; either may be NULL.  accumulate != 0 adds
 *        to what is there, 0 overwrites.
 * gamma NULL: ones. */
int adacomp_norm_backward(const adacomp_norm_t *norm, const void *dy, const void *dz_add, const void *z, const float *mean,
                          const float *rstd, const float *gamma, const adacomp_dropout_t *dropout, void *dz, void *dx,
                          float *dgamma, float *dbeta, int accumulate, void *workspace, size_t workspace_bytes,
                          void *hip_stream);

/* ---- softmax with a learned relative position bias ------------------------------------------------ */

#define ADACOMP_BIAS_DISTANCE_MAX 2048u

/* The usual map of distances to buckets, for max_distance D a HOST array of 2 D + 1 numbers: map[d + D] for
 * d = key - query in -D .. D, and the ends for everything beyond.  With both directions one half of the
 * buckets is for keys behind the query (d > 0); else those all have bucket 0.  Of the n buckets of a
 * direction the first n / 2 are for single distances, the others up to D spaced logarithmically:
 * n / 2 + floor(log(|d| / (n / 2)) / log(D / (n / 2)) (n - n / 2)), at most n - 1; quotients within 1e-9 below
 * a whole number count as that number.  n_buckets at least 2 (4 with both directions, and even),
 * max_distance above n / 2 and up to ADACOMP_BIAS_DISTANCE_MAX.  Any other map can be used as well. */
int adacomp_relative_buckets(uint32_t n_buckets, uint32_t max_distance, int both_directions, int32_t *map);

/* Scores [batch, heads, queries, keys], query i of batch b standing at position
 * (query_starts ? query_starts[b] : query_start) + i, key j at position j.
 * A place is admitted if j < key_lengths[b] (with key_lengths), j <= the query's position (with causal),
 * and mask[b, h, i, j] != 0 (with mask).  What stands in other places is never looked at.
 *   t = scale * score + table[map[clamp(j - position, -D, D) + D], head], a float32: only scores and products beyond its range
 *       are infinities (a row of a type's lowest value is even at a scale of 1, not empty)
 *   P = exp(t - lse), lse = log(sum over the row's admitted places of exp(t)); a row without any (or with
 *       -infinity in all of them) has P = 0 and lse = -infinity
 * table      [n_buckets, heads] float32;  map  2 max_distance + 1 device int32, clamped to 0 .. n_buckets - 1
 * batch heads queries < 2^31, heads up to 2^20, keys < 2^30; max_distance 1 .. ADACOMP_BIAS_DISTANCE_MAX;
 * n_buckets 1 .. 2 ADACOMP_BIAS_DISTANCE_MAX + 1.
 * Strides of the mask may be 0 (one mask for several heads, say). */
typedef struct {
    const void *data;
    int64_t batch_stride, head_stride, row_stride;
} adacomp_view_t;

typedef struct {
    uint32_t batch, heads, queries, keys, dtype, causal;
    uint32_t n_buckets, max_distance;
    float scale;
    int32_t query_start;
    const int32_t *query_starts; /* device [batch] or NULL */
    const int32_t *key_lengths;  /* device [batch] or NULL */
    const float *table;
    const int32_t *map;
    adacomp_view_t mask;         /* uint8; data NULL: no mask */
} adacomp_bias_softmax_t;

/* Bytes of workspace of the two calls below.  Nothing in it is kept between calls. */
size_t adacomp_bias_softmax_workspace_bytes(uint32_t batch, uint32_t heads, uint32_t queries, uint32_t keys,
                                            uint32_t max_distance);

/* probs = D(P), zeros where not admitted; the generator's row is (b heads + h) queries + i, its column j.
 * lse [batch, heads, queries] contiguous float32, or NULL.  dropout may be NULL. */
int adacomp_bias_softmax_forward(const adacomp_bias_softmax_t *op, const adacomp_view_t *scores, const adacomp_view_t *probs,
                                 float *lse, const adacomp_dropout_t *dropout, void *workspace, size_t workspace_bytes,
                                 void *hip_stream);

/* From the scores, the lse of the forward pass and dprobs, the gradient of probs:
 *   dP = D(dprobs);  e = P (dP - sum over the row of P dP);  dscores = scale e, zeros where not admitted;
 *   dtable[k, h] = sum of e over all places of head h whose distance has bucket k.
 * dtable [n_buckets, heads] may be NULL; accumulate != 0 adds to what is there, 0 overwrites.
 * The same op and dropout as in the forward pass.  lse is a float32, and P as exact as that allows: where it is beyond 2^22 in
 * magnitude (rows of a type's lowest value, say) P is 1 at the places that are as near to it as its rounding. */
int adacomp_bias_softmax_backward(const adacomp_bias_softmax_t *op, const adacomp_view_t *scores, const float *lse,
                                  const adacomp_view_t *dprobs, const adacomp_dropout_t *dropout,
                                  const adacomp_view_t *dscores, float *dtable, int accumulate, void *workspace,
                                  size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
