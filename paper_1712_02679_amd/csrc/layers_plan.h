// layers_plan.h -- what the checks (layers_api.hip) and the kernels (layers_norm.hip, layers_softmax.hip) of the calls in
// adacomp_layers.h share: kernel arguments and the rules that choose a kernel's form.
#pragma once

#include <algorithm>
#include <cstdint>

#include "adacomp_layers.h"
#include "adacomp_plan.h"

namespace adacomp {

// Dropout as the kernels take it.  on == 0: none (also p so small that its threshold is 0).
struct DropArgs {
    const uint64_t *step;
    uint32_t seed_lo, seed_hi, stream_lo, stream_hi;
    uint32_t on, threshold;   // kept where a 16-bit number is at least threshold
    float factor;
};

constexpr uint64_t kInputsPast = uint64_t(192) << 20;   // bytes of 16-bit inputs that go past the caches, where their rows are whole lines

// A thread takes groups of 8 columns, each one counter of the generator: threads to a row (a part of a wave, a wave, or a
// workgroup) times groups to a thread cover the row.
struct RowForm {
    uint32_t threads, groups;
    uint32_t teams() const { return threads > 256u ? 1u : 256u / threads; }   // rows that a workgroup has in hand
    uint32_t workgroup() const { return std::max(threads, 256u); }
};

struct DropoutLaunch {
    const void *x, *residual;
    void *y;
    uint64_t x_stride, residual_stride, y_stride, first_row;
    uint32_t rows, cols, groups;   // groups to a row
    uint32_t dtype;
    DropArgs drop;
};

struct NormForward {
    const void *x, *residual;
    const float *gamma, *beta;
    void *z, *y;
    float *mean, *rstd;
    uint64_t x_stride, residual_stride, z_stride, y_stride;
    uint64_t all_rows, first_row;   // of the call; of a launch, whose pointers begin there
    uint32_t rows, cols;
    float eps;
    DropArgs drop;
};

struct NormBackward {
    const void *dy, *dz_add, *z;
    const float *mean, *rstd, *gamma;
    void *dz, *dx;
    float *partial;   // [workgroups][2][pitch]: sums of dy h and of dy over the rows of a workgroup
    uint64_t dy_stride, dz_add_stride, z_stride, dz_stride, dx_stride;
    uint32_t rows, cols, pitch;
    DropArgs drop;
};

struct NormReduce {
    const float *partial;
    float *dgamma, *dbeta;
    uint32_t parts, pitch, cols, accumulate;
};

// Threads to a row of the forward pass: 16 values to a thread, or up to 32 in the widest rows (16 and not 8: twice the bytes on their way for a
// wave, at no more than 64 registers).
inline uint32_t norm_forward_threads(uint32_t cols)
{
    uint32_t threads = 8;
    while (threads < 1024u && threads * (cols <= 64u ? 8u : 16u) < cols) threads *= 2u;
    return threads;
}
// Rows of one of its launches, which has at most 2^31 threads: the grid is counted in threads, in 32 bits.
inline uint64_t norm_forward_rows(const RowForm &row) { return std::min(uint64_t(1) << 22, row.teams() * ((uint64_t(1) << 31) / row.workgroup())); }

uint32_t norm_parts(uint64_t rows, uint32_t cols);   // workgroups of the backward pass
inline uint32_t norm_pitch(uint32_t cols) { return (cols + 7u) & ~7u; }

int launch_dropout(const DropoutLaunch &a, void *stream);
int launch_norm_forward(const NormForward &a, uint32_t dtype, void *stream);
int launch_norm_backward(const NormBackward &a, uint32_t dtype, uint32_t parts, void *stream);
int launch_norm_reduce(const NormReduce &a, void *stream);

struct ViewArgs {
    const void *data;
    int64_t batch, head, row;
};

// One launch over the rows of a call, or over parts of its rows.
struct SoftmaxArgs {
    ViewArgs scores, in, out, mask;   // in: dprobs
    const int32_t *query_starts, *key_lengths, *map;
    const float *table;
    float *lse;         // written by the forward pass, read by the backward pass
    float *part_stats;  // [rows][parts][2], of a row cut into parts: (maximum, sum) or (sum of P dP, -)
    float *bias_sums;   // [heads][groups][places]: sums of e by distance, of a workgroup's rows
    uint32_t batch, heads, queries, keys, causal;
    uint32_t n_buckets, distance;
    uint32_t first_place, places;   // of the map's 2 D + 1 entries, those that the call can need
    int32_t query_start;
    float scale;
    uint32_t rows_per_wg, wgs_per_head;   // forward: consecutive rows of a workgroup, workgroups to a (batch, head), or merged to a head; backward: workgroups to a head
    uint32_t row_parts;                   // parts of a row
    uint32_t merged;                      // forward: workgroups share out a head's rows of all sequences, not of one
    DropArgs drop;
};

struct BiasReduce {
    const float *bias_sums;
    const int32_t *map;   // at the first place
    float *dtable;
    uint32_t heads, groups, places, n_buckets, accumulate;
};

// How a call goes: whole rows, or rows cut into parts (two launches)
struct SoftmaxForm {
    RowForm row;
    uint32_t parts;   // 1: whole rows
};
SoftmaxForm softmax_form(uint32_t keys, uint32_t places, bool backward);
// Most workgroups to a head that the backward pass takes in a form; in any form, at most a row each and this many in all.
constexpr uint32_t kMostResident = 6;   // workgroups on a compute unit; of kernels of which 7 should fit, 6 are faster (16 x 1000 x 1000 x 16 bf16 309 / 373 us)
uint32_t softmax_back_groups_most(uint64_t rows_of_head, uint32_t heads, const SoftmaxForm &form);

int launch_softmax_forward(const SoftmaxArgs &a, uint32_t dtype, const SoftmaxForm &form, void *stream);
int launch_softmax_backward(const SoftmaxArgs &a, uint32_t dtype, const SoftmaxForm &form, uint32_t &groups, void *stream);   // groups: workgroups to a head, of the bias_sums
int launch_bias_reduce(const BiasReduce &a, void *stream);

}  // namespace adacomp
