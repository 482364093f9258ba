// sequence_plan.h -- what the checks (sequence_api.hip) and the kernels (sequence_embed.hip, sequence_recurrence.hip,
// sequence_distill.hip) of the calls in adacomp_sequence.h share: kernel arguments and the rules that choose a kernel's form.
#pragma once

#include "adacomp_sequence.h"
#include "layers_plan.h"

namespace adacomp {

// ---- embedding ----------------------------------------------------------------------------------------------------

struct EmbedPlace { uint32_t token, row; };   // a row of the call, in the order of the tokens

struct EmbedArgs {
    const void *tokens;
    const float *table;   // forward
    void *rows_of;        // y, or dy
    float *dtable;        // backward
    uint32_t *first;      // [vocab + 1]: where a token's places begin in order
    EmbedPlace *order;    // [rows]: places, sorted by token and then by row
    float *parts;         // [pieces][2][pitch]
    uint64_t stride, first_row;
    uint32_t rows, vocab, cols, groups;   // groups of 8 to a row
    uint32_t index64, accumulate;
    uint32_t range, team, slabs, piece, pieces, pitch;   // see EmbedForm
    uint32_t zero_team;   // threads that write a row of zeros
    float scale;
    DropArgs drop;
};

constexpr uint32_t kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr uint32_t kSortRange = 512;   // most tokens of a sorting workgroup, which has a count of each for every wave in LDS

// How a backward pass goes.
struct EmbedForm {
    uint32_t range;    // tokens of a sorting workgroup
    uint32_t team;     // threads to a row, 8 columns each
    uint32_t slabs;    // of a row, if it has more columns than a team takes
    uint32_t piece;    // places that are added up together
    uint32_t pieces, pitch;
};

inline EmbedForm embed_form(uint32_t rows, uint32_t vocab, uint32_t cols)
{
    EmbedForm f = {};
    f.range = std::min(kSortRange, (vocab + kComputeUnits - 1u) / kComputeUnits);
    f.team = 8;
    while (f.team < 256u && f.team * 8u < cols) f.team *= 2u;
    f.slabs = (cols + f.team * 8u - 1u) / (f.team * 8u);
    // as long as there are waves for all compute units
    f.piece = 64;
    while (f.piece > 8u && uint64_t(rows) * f.slabs * f.team / (uint64_t(f.piece) * 64u) < 8u * kComputeUnits) f.piece /= 2u;
    f.pieces = (rows + f.piece - 1u) / f.piece;
    f.pitch = (cols + 7u) & ~7u;
    return f;
}

int launch_embed_forward(const EmbedArgs &a, uint32_t dtype, void *stream);
int launch_embed_backward(const EmbedArgs &a, uint32_t dtype, void *stream);

// ---- gated linear recurrence --------------------------------------------------------------------------------------

struct StepsArgs {
    const void *data;
    int64_t batch, row;
};

struct RecurrenceArgs {
    StepsArgs x, forget, out;
    StepsArgs y;                        // forward: y, backward: dy
    StepsArgs dx, dforget, dout;
    const float *bias, *first;          // first: forward: h[-1], backward: dlast
    float *last;                        // forward: the last state, backward: dfirst
    float *states;
    float *dbias_parts;                 // [batch][segments][channels]
    float *changes;                     // [batch][segments][2][channels]: what a part does to the state
    const int32_t *lengths;
    const uint8_t *resets;
    int64_t resets_stride;
    uint32_t batch, length, channels, slabs;   // slabs of kSlab channels
    uint32_t kept;                             // states of a sequence
    uint32_t segments, segment;                // parts of a sequence, places of a part
    uint32_t first_sequence;                   // of a launch
    uint32_t near_rows;                        // rows of all tensors are so near that a wave's lie within 32 bits
    uint32_t apart;                            // results share no memory with what is read
};

constexpr uint32_t kSlab = 64;   // channels of a workgroup: a line of memory in 16 bits

// Into how many parts a sequence is cut, and how many places a part has: one where every compute unit has a workgroup anyway, as parts are read
// twice; otherwise as many as give two (8 x 2048 x 2048 bf16, 256 workgroups, in one / two parts: 53 / 76 us, backward 133 / 144; 4 x 2048 x 2048 in two /
// four / eight: 53 / 41 / 43 us, backward 101 / 75 / 77).
struct RecurrenceForm { uint32_t segments, segment; };
inline RecurrenceForm recurrence_form(uint32_t batch, uint32_t length, uint32_t channels)
{
    constexpr uint32_t kLeast = 128;   // places of a part, whole blocks of a workgroup (128 / 256: 1 x 1024 x 512 13.6 / 17.6 us, backward 20 / 30)
    const uint64_t workgroups = uint64_t(batch) * ((channels + kSlab - 1u) / kSlab);
    if (workgroups == 0 || workgroups >= kComputeUnits || length == 0) return {1u, std::max(length, 1u)};
    const uint64_t wanted = std::min<uint64_t>((2u * kComputeUnits + workgroups - 1u) / workgroups, (length + kLeast - 1u) / kLeast);
    const uint32_t segment = std::max<uint32_t>(1u, uint32_t(length / wanted + kLeast / 2u) / kLeast) * kLeast;
    return {(length + segment - 1u) / segment, segment};
}

// Sequences of a launch of workgroups of up to kRecurrenceThreads, `of_one` of them to a sequence: a grid is counted in threads, in 32 bits.
constexpr uint32_t kRecurrenceThreads = 512;
constexpr uint32_t recurrence_sequences(uint32_t of_one) { return (1u << 31) / kRecurrenceThreads / of_one; }

struct BiasSumArgs {
    const float *parts;
    float *dbias;
    uint32_t count, channels, accumulate;
};

int launch_recurrence_forward(const RecurrenceArgs &a, uint32_t dtype, void *stream);
int launch_recurrence_backward(const RecurrenceArgs &a, uint32_t dtype, void *stream);
int launch_bias_sum(const BiasSumArgs &a, void *stream);

// ---- distillation -------------------------------------------------------------------------------------------------

struct DistillArgs {
    const void *logits;
    void *dlogits;
    const void *teacher_tokens, *teacher_logits, *targets;
    float *loss, *lse;          // lse: written by the forward pass, read by the backward pass
    const float *dloss;
    uint64_t logits_stride, dlogits_stride, tokens_stride, teacher_stride;
    uint64_t rows;
    uint32_t vocab, top;
    uint32_t tokens64, targets64, teacher_dtype;
    float per_temperature, hard;    // 1 / temperature
    float soft_loss, soft_grad;     // soft temperature^2 of a loss, soft temperature of a gradient
    float scale;
};

// Threads to a row, groups of 8 logits to a thread, whether a row is held in registers.  Short rows are held, with the entries of all teams within 64 KB of
// LDS: rows of up to 256 logits have forms of their own, which alone look whether a row has 8 (in the form for up to 1024 that look costs 32768 x 300 bf16
// 22.3 / 22.9 us, losses).  Others are read in parts, twice for loss and gradient: held in registers they leave so few waves that rows of 16384 take
// twice as long.  A wave to a row needs no barrier, but many rows; few long rows need all threads that a workgroup can have.
// 64 / 256 / 1024 threads, loss and gradient of bf16 with 64 top tokens, us: 32768 x 2000 91 / 176 / 840, 16384 x 5000 100 / 128 / 430, 8192 x 16384
// 166 / 141 / 249, 4096 x 65536 331 / 288 / 298, 1024 x 5000 18.7 / 18.5 / 34, 256 x 50000 65 / 27 / 23.
struct DistillForm {
    uint32_t threads, groups, held;
    constexpr bool short_rows() const { return held != 0u && threads * groups == 32u; }   // rows may have fewer than 8 logits
};
constexpr DistillForm distill_form(uint64_t rows, uint32_t vocab, uint32_t top)
{
    if (vocab <= 256u && top < 160u) return {8u, 4u, 1u};
    if (vocab <= 256u) return {32u, 1u, 1u};
    if (vocab <= 1024u) return {32u, 4u, 1u};
    if (rows >= 4096u && vocab <= 8192u) return {64u, 2u, 0u};
    if (rows >= 512u || vocab <= 16384u) return {256u, 2u, 0u};
    return {1024u, 2u, 0u};
}

enum DistillPass { LOSS, LOSS_GRAD, GRAD };
int launch_distill(const DistillArgs &a, uint32_t dtype, DistillPass pass, void *stream);

}  // namespace adacomp
