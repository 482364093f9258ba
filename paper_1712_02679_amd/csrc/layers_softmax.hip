// layers_softmax.hip -- kernels of the masked softmax with a learned relative position bias (adacomp_layers.h).
//
// The bias of a place depends on its head and on clamp(key - query, -D, D) alone, so a workgroup, whose rows all belong to one
// head, lays out the head's values in LDS once, for the distances that the call can have, and a place costs one LDS read; groups of 8 keys that lie
// beyond D on one side cost none.  The gradient goes the same way back: sums by distance, added up in LDS (inside a row all
// distances differ, so no two threads of a row meet, and rows follow each other), those beyond D in registers; k_bias_reduce
// adds the workgroups' sums and only then turns distances into buckets.
//
// Forward reads the admitted scores and writes all probabilities, backward reads scores and dprobs and writes dscores, once each;
// a row of up to 32768 keys stays in registers between its reductions.  Measured, bf16, 4 x 16 x 2048 x 2048 with dropout: forward 197 us (5.5 TB/s),
// causal 163 us (4.9 TB/s of what it needs), backward 319 us (5.1 TB/s), with padding 293.  What bounds the large calls is memory, and in the backward
// pass also the vector units: 340 instructions for 8 values of a wave's threads, 55 of them the generator's (padded, without dropout 273 us).
// Short rows are far from that, bound by what a row costs whatever its length (with dropout: forward 8000 x 16 x 17 x 17 162 us, 1.0 TB/s, 512 x 16 x
// 100 x 100 107 us, 3.1; backward 2048 x 16 x 30 x 30 117 us, 1.6), and so is the backward pass where many distances leave few rows to a
// workgroup (32 x 16 x 1500 x 400 with distances up to 800 643 us, 2.9 TB/s).  The kernels use all of their scalar registers, and keep 9 to 92 more values in lanes
// of vector registers; none has vector registers in memory.
#include <atomic>

#include "layers_device.h"

namespace adacomp {

constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = float(1.4426950408889634 - double(kLog2e)), kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();

// The bias by distance index x = key - query + D, as far as a call can have that distance (a.places of them from a.first_place on), and the sums of its
// gradient, lie in LDS with 8 more places at either end, so that a group of 8 keys that reaches over an end needs no clamp.  Place X = x + 8 is in cell X + X / 8: neighbouring lanes are 8 places
// and so 9 cells apart, in different banks.  Groups begin at multiples of 8 keys, so X % 8 is the same for a whole row.
constexpr uint32_t kGuard = 8;
__host__ __device__ constexpr uint32_t cell(uint32_t X) { return X + (X >> 3); }
__host__ __device__ constexpr uint32_t cells(uint32_t places) { return (cell(places - 1u + 2u * kGuard) + 3u) & ~3u; }

// Exponents are in natural units, as in the formula, so that they are finite wherever scale * score is: in units of log2 the lowest
// bf16 value would be -infinity at a scale of 1.  16-bit tensors: the product with log2(e) is rounded, 5e-7 of the result at most where the
// argument is about 10, far below their own rounding.  32-bit ones: that rounding is made good to first order (6 x 5 x 333 x 777: dscores
// 3.1e-7 -> 2.3e-7 off).
template <typename T> __device__ __forceinline__ float exp_of(float x)
{
    const float y = x * kLog2e, p = __builtin_amdgcn_exp2f(y);
    if constexpr (sizeof(T) == 2) return p;
    const float off = fabsf(x) < 200.f ? fmaf(x, kLog2e, -y) + x * kLog2eRest : 0.f;   // infinities have none
    return fmaf(p, off * kLn2, p);
}

// A workgroup's copy of its head's bias.
__device__ __forceinline__ void stage_bias(float *bias, const SoftmaxArgs &a, uint32_t head)
{
    const int last = int(a.places) - 1;
    for (int X = threadIdx.x; X <= last + 2 * int(kGuard) - 1; X += blockDim.x) {
        const int32_t b = min(max(a.map[a.first_place + min(max(X - int(kGuard), 0), last)], 0), int32_t(a.n_buckets) - 1);
        bias[cell(X)] = a.table[uint64_t(b) * a.heads + head];
    }
}

// What a row looks at.
struct Row {
    const uint8_t *mask;   // NULL: none
    int limit;             // keys below it are admitted, as far as the mask goes
    int shift;             // place of key j: j + shift
};

__device__ __forceinline__ Row row_of(const SoftmaxArgs &a, uint32_t b, uint32_t h, uint32_t i)
{
    Row r;
    const int64_t at = int64_t(a.query_starts ? a.query_starts[b] : a.query_start) + i;
    int64_t limit = a.keys;
    if (a.key_lengths) limit = min(limit, int64_t(a.key_lengths[b]));
    if (a.causal) limit = min(limit, at + 1);
    r.limit = int(max(limit, int64_t(0)));
    // keys are below 2^30: a shift beyond these bounds is beyond D for every key either way
    r.shift = int(min(max(int64_t(a.distance + kGuard - a.first_place) - at, -(int64_t(1) << 30) - 8192), int64_t(1) << 30));
    r.mask = a.mask.data ? static_cast<const uint8_t *>(a.mask.data) + int64_t(b) * a.mask.batch + int64_t(h) * a.mask.head + int64_t(i) * a.mask.row : nullptr;
    return r;
}

// Where a group of 8 keys from j on lies.
struct Window {
    int X;          // place of its first key
    uint32_t base;  // cell of the multiple of 8 at or below X, if any of the 8 lies between the ends
    __device__ __forceinline__ Window(const Row &r, int j) : X(j + r.shift), base(uint32_t(9 * (X >> 3))) {}
    __device__ __forceinline__ bool above(int last) const { return X >= last + int(kGuard); }
    __device__ __forceinline__ bool below() const { return X <= 0; }
    // cell of key k of the group: base + X % 8 + k, and one more behind a multiple of 8
    __device__ __forceinline__ uint32_t of(const Row &r, int k) const
    {
        const uint32_t in = (uint32_t(r.shift) & 7u) + uint32_t(k);
        return base + (in + (in >> 3));
    }
};

// The admitted ones of 8 keys, a bit each, of which n are below the row's limit; mask: their bytes of the mask.
template <bool MASK> __device__ __forceinline__ uint32_t admitted8(uint64_t mask, int n)
{
    uint32_t bits = n >= 8 ? 0xFFu : (1u << max(n, 0)) - 1u;
    if constexpr (MASK) {
        uint32_t keep = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) keep |= (uint32_t(mask >> (8 * k)) & 0xFFu) ? 1u << k : 0u;
        bits &= keep;
    }
    return bits;
}

// The mask's bytes for the groups of a row; ones without a mask.
template <typename T, int TPR, int V, int FLOW, bool SHORT>
__device__ __forceinline__ void load_mask(const RowGroups<T, TPR, V, FLOW, SHORT> &groups, raw8<uint8_t> (&mask)[V], const Row &r)
{
    if (r.mask) RowGroups<uint8_t, TPR, V, CACHED, SHORT>{groups.t, groups.cols, groups.first}.load_below(mask, r.mask, uint32_t(r.limit));
    else
#pragma unroll
        for (int v = 0; v < V; ++v) mask[v] = raw8<uint8_t>(uint8_t(1));
}

// The mask's bytes that were loaded for round v, in their place.
template <typename G> __device__ __forceinline__ uint64_t mask_of(const G &groups, raw8<uint8_t> raw, int v)
{
    const uint64_t m = __builtin_bit_cast(uint64_t, raw);
    return groups.ends_in(v) && !(G::kShort && groups.cols < 8u) && groups.ends_here() ? m >> 8u * (8u - groups.cols % 8u) : m;
}

// scale * s + bias - less of 8 keys.
__device__ __forceinline__ f32x8 biased8(f32x8 s, const SoftmaxArgs &a, float scale, const Row &r, const Window &w, const float *bias, float low, float high, float less)
{
    f32x8 t;
    const int last = int(a.places) - 1;
    if (w.above(last) || w.below()) {
        const float b = (w.below() ? low : high) - less;
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = fmaf(s[k], scale, b);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = fmaf(s[k], scale, bias[w.of(r, k)] - less);
    }
    return t;
}

// WHOLE: a row at a time.  STATS, WRITE: a part of a row, first its maximum and sum, then, from those of all parts, the results.
enum Phase { WHOLE, STATS, WRITE };
// MASKED: with a mask.  SHORT: rows shorter than a group, with or without one, in forms of more than 8 threads to a row, which only the
// backward pass gives to such rows, where the distances are many.
// ONCE: large inputs without a mask, in whole lines, past the caches.
// MERGED, without a mask and with one: workgroups of the forward pass share out a head's rows of all sequences instead of one sequence's.
enum Kind { PLAIN, MASKED, SHORT, ONCE, MERGED, MERGED_MASKED };
template <int KIND> constexpr bool kMasked = KIND == MASKED || KIND == SHORT || KIND == MERGED_MASKED;
template <int KIND> constexpr bool kMerged = KIND == MERGED || KIND == MERGED_MASKED;

// ---- forward ------------------------------------------------------------------------------------------------------

template <typename T, int TPR, int V, int PHASE, int KIND> __global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_softmax_forward(SoftmaxArgs a)
{
    constexpr uint32_t TEAMS = TPR > 256 ? 1 : 256 / TPR;
    constexpr int LANES = TPR > 64 ? 64 : TPR;
    extern __shared__ float bias[];
    __shared__ float room[2][2][16];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>();
    const Drop d = drop_of(a.drop);
    uint32_t turn = 0;
    const uint64_t blocks = uint64_t(kMerged<KIND> ? 1u : a.batch) * a.heads * a.wgs_per_head * a.row_parts;
    for (uint64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
        uint32_t unit = uint32_t(block), part = 0;
        if constexpr (PHASE != WHOLE) { unit = uint32_t(block / a.row_parts); part = uint32_t(block - uint64_t(unit) * a.row_parts); }
        const uint32_t bh = unit / a.wgs_per_head, first = (unit - bh * a.wgs_per_head) * a.rows_per_wg;
        uint32_t b = kMerged<KIND> ? 0u : bh / a.heads;
        const uint32_t h = bh - b * a.heads;
        const T *scores = static_cast<const T *>(a.scores.data) + int64_t(b) * a.scores.batch + int64_t(h) * a.scores.head;
        T *out = static_cast<T *>(const_cast<void *>(a.out.data)) + int64_t(b) * a.out.batch + int64_t(h) * a.out.head;
        const uint32_t base = part * (TPR * V * 8u), end = min(first + a.rows_per_wg, kMerged<KIND> ? a.batch * a.queries : a.queries);
        raw8<T> raw[V];
        raw8<uint8_t> mask[V];
        Row next = {};
        auto fetch = [&](uint32_t i) {   // a row's scores are on their way while the one before is worked on, the first one's while the bias is laid out
            const T *s = scores;
            if constexpr (kMerged<KIND>) {
                b = i / a.queries;
                i -= b * a.queries;
                s += int64_t(b) * a.scores.batch;
            }
            next = row_of(a, b, h, i);
            const RowGroups<T, TPR, V, KIND == ONCE ? int(ALL_PAST) : kFlow<T>, TPR == 8 || KIND == SHORT> groups = {again(t), again_uniform(a.keys), base};
            groups.load_below(raw, s + int64_t(i) * a.scores.row, uint32_t(next.limit));
            if constexpr (kMasked<KIND>) load_mask(groups, mask, next);
        };
        if (first + team < end) fetch(first + team);
        if (block != blockIdx.x) __syncthreads();   // the rows before are done with the bias
        stage_bias(bias, a, h);
        __syncthreads();
        const float low = bias[0], high = bias[cell(a.places - 1u + kGuard)];
        for (uint32_t i = first + team; i < end; i += TEAMS) {
            const Row r = next;
            uint64_t row = uint64_t(bh) * a.queries + i;
            T *o = out + int64_t(i) * a.out.row;
            if constexpr (kMerged<KIND>) {
                const uint32_t q = i - b * a.queries;
                row = (uint64_t(b) * a.heads + h) * a.queries + q;
                o = out + int64_t(b) * a.out.batch + int64_t(q) * a.out.row;
            }
            const RowGroups<T, TPR, V, KIND == ONCE ? int(ALL_PAST) : kFlow<T>, TPR == 8 || KIND == SHORT> groups = {again(t), again_uniform(a.keys), base};
            const Drop dr = again(d);
            f32x8 p[V];
            uint32_t bits = 0;   // admitted places, 8 to a group
            float m = -kInf;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int j = int(groups.col(v)), n = r.limit - j;
                // rounds of which a wave has nothing are left out; its other threads go along, and have nothing admitted
                p[v] = -kInf;
                if (__any(n > 0)) {
                    const uint32_t here = admitted8<kMasked<KIND>>(kMasked<KIND> ? mask_of(groups, mask[v], v) : 0, n);
                    bits |= here << (8 * v);
                    p[v] = biased8(groups.values(raw[v], v), a, a.scale, r, Window(r, j), bias, low, high, 0.f);
                    if (here != 0xFFu) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) p[v][k] = here >> k & 1u ? p[v][k] : -kInf;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) m = fmaxf(m, p[v][k]);
                }
            }
            if (i + TEAMS < end) fetch(i + TEAMS);
            // exponentials from the maximum of a wave's lanes; the waves' sums are joined behind them
            m = over_lanes<Max, LANES>(m);
            const float from = m == -kInf ? 0.f : m;
            // 16 bits: units of log2 in the same operation as the difference (a product of its own costs 2 %).  The rounding of from * unit is common to the
            // wave's values, and no larger than that of its maximum; beyond 2^24 scores that differ at all differ by thousands, in any unit, and the
            // product could overflow.
            const float unit = fabsf(from) < 0x1p24f ? kLog2e : 1.f, from_units = from * unit;
            float l = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (__any(bits >> (8 * v) & 0xFFu)) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        p[v][k] = sizeof(T) == 2 ? __builtin_amdgcn_exp2f(fmaf(p[v][k], unit, -from_units)) : exp_of<T>(p[v][k] - from);
                        l += p[v][k];
                    }
                }
            l = over_lanes<Add, LANES>(l);
            float top = m, total = l;
            if constexpr (TPR > 64) {
                if (threadIdx.x % 64u == 0u) { room[turn][0][threadIdx.x / 64u] = m; room[turn][1][threadIdx.x / 64u] = l; }
                __syncthreads();
                top = -kInf;
#pragma unroll
                for (int w = 0; w < TPR / 64; ++w) top = fmaxf(top, room[turn][0][w]);
                const float from_top = top == -kInf ? 0.f : top;
                total = 0.f;
#pragma unroll
                for (int w = 0; w < TPR / 64; ++w) total = fmaf(room[turn][1][w], exp_of<T>(room[turn][0][w] - from_top), total);
                turn ^= 1u;
            }
            if constexpr (PHASE == STATS) {
                if (threadIdx.x == 0u) {
                    float *to = a.part_stats + (row * a.row_parts + part) * 2u;
                    to[0] = top;
                    to[1] = total;
                }
                continue;
            }
            if constexpr (PHASE == WRITE) {
                const float *of = a.part_stats + row * a.row_parts * 2u;
                top = -kInf;
                for (uint32_t q = 0; q < a.row_parts; ++q) top = fmaxf(top, of[2u * q]);
                const float from_top = top == -kInf ? 0.f : top;
                total = 0.f;
                for (uint32_t q = 0; q < a.row_parts; ++q) total = fmaf(of[2u * q + 1u], exp_of<T>(of[2u * q] - from_top), total);
            }
            // a wave of nothing but -infinity has zeros, whatever the row's maximum; a row's NaN is in its total
            float factor = total == 0.f ? 0.f : (m == -kInf ? 1.f : exp_of<T>(from - top)) / total;
            if (a.drop.on) factor *= d.factor;
            if (a.lse && t == 0u && part == 0u) a.lse[row] = total == 0.f ? -kInf : sizeof(T) == 2 ? fmaf(log2f(total), kLn2, top) : top + logf(total);
            groups.store(o, [&](int v) {
                f32x8 y = {};
                const uint32_t here = bits >> (8 * v) & 0xFFu;
                if (__any(here != 0u)) {
                    y = p[v] * factor;
                    if (here != 0xFFu) {   // a row's NaN stays where it looks
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = here >> k & 1u ? y[k] : 0.f;
                    }
                    if (a.drop.on) y = kept8(y, dr, groups.col(v) / 8u, uint32_t(row));
                }
                return y;
            });
        }
    }
}

// ---- backward -----------------------------------------------------------------------------------------------------

template <typename T, int TPR, int V, int PHASE, int KIND> __global__ __launch_bounds__(TPR > 256 ? TPR : 256, 4) void k_softmax_backward(SoftmaxArgs a)
{
    constexpr uint32_t TEAMS = TPR > 256 ? 1 : 256 / TPR, WG = TPR > 256 ? TPR : 256;
    constexpr int LANES = TPR > 64 ? 64 : TPR;
    extern __shared__ float lds[];
    __shared__ float room[2][16];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>();
    const uint32_t size = cells(a.places);
    const int last = int(a.places) - 1;
    float *bias = lds, *acc = lds + size * (1u + team);   // every team has sums of its own
    const bool sums = PHASE != STATS && a.bias_sums;
    const uint32_t h = blockIdx.x / a.wgs_per_head, group = blockIdx.x - h * a.wgs_per_head;
    const Drop d = drop_of(a.drop);
    const float up_factor = a.drop.on ? d.factor : 1.f;
    stage_bias(bias, a, h);
    if (sums)
        for (uint32_t x = threadIdx.x; x < size * TEAMS; x += WG) lds[size + x] = 0.f;
    __syncthreads();
    const float bias_low = bias[0], bias_high = bias[cell(uint32_t(last) + kGuard)];
    float low = 0.f, high = 0.f;   // sums of e beyond the ends of the map
    const uint64_t units = uint64_t(a.batch) * a.queries * a.row_parts;
    uint32_t turn = 0;
    for (uint64_t unit = uint64_t(group) * TEAMS + team; unit < units; unit += uint64_t(a.wgs_per_head) * TEAMS) {
        uint32_t row_of_head = uint32_t(unit), part = 0;
        if constexpr (PHASE != WHOLE) { row_of_head = uint32_t(unit / a.row_parts); part = uint32_t(unit - uint64_t(row_of_head) * a.row_parts); }
        const uint32_t b = row_of_head / a.queries, i = row_of_head - b * a.queries;
        const uint32_t base = part * (TPR * V * 8u);
        const Row r = row_of(a, b, h, i);
        const uint64_t row = (uint64_t(b) * a.heads + h) * a.queries + i;
        const T *s = static_cast<const T *>(a.scores.data) + int64_t(b) * a.scores.batch + int64_t(h) * a.scores.head + int64_t(i) * a.scores.row;
        const T *up = static_cast<const T *>(a.in.data) + int64_t(b) * a.in.batch + int64_t(h) * a.in.head + int64_t(i) * a.in.row;
        T *o = static_cast<T *>(const_cast<void *>(a.out.data)) + int64_t(b) * a.out.batch + int64_t(h) * a.out.head + int64_t(i) * a.out.row;
        const uint32_t keys = again_uniform(a.keys);
        const RowGroups<T, TPR, V, KIND == ONCE ? int(ALL_PAST) : kFlow<T>, TPR == 8 || KIND == SHORT> groups = {again(t), keys, base};
        const Drop dr = again(d);
        raw8<T> raw[V], raw_up[V];
        groups.load_below(raw, s, uint32_t(r.limit));
        groups.load_below(raw_up, up, uint32_t(r.limit));
        raw8<uint8_t> mask[V];
        if constexpr (kMasked<KIND>) load_mask(groups, mask, r);
        const float lse = a.lse[row], from = lse == -kInf ? kInf : lse;
        // Beyond 2^22 an lse has no fraction left, and its roundings alone would make exponents of any size: there, places that are as
        // near to it as that have P = 1 (rows of the type's lowest value, say; their number is lost in lse).
        const bool coarse = !(fabsf(from) < 4194304.f);
        const float less = coarse || sizeof(T) == 4 ? 0.f : from;
        f32x8 p[V], dp[V];
        uint32_t admitted = 0;   // 8 places to a group
        float inner = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int j = int(groups.col(v)), n = r.limit - j;
            p[v] = 0.f;
            dp[v] = 0.f;
            if (__any(n > 0)) {   // rounds of which a wave has nothing are left out; its other threads go along, and have nothing admitted
                const uint32_t bits = admitted8<kMasked<KIND>>(kMasked<KIND> ? mask_of(groups, mask[v], v) : 0, n);
                admitted |= bits << (8 * v);
                p[v] = biased8(groups.values(raw[v], v), a, a.scale, r, Window(r, j), bias, bias_low, bias_high, less);
                if (sizeof(T) == 4 && !coarse) {   // the difference as the formula has it: exact where it is small
#pragma unroll
                    for (int k = 0; k < 8; ++k) p[v][k] -= from;
                }
                if (coarse) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float x = p[v][k] - from;
                        p[v][k] = x > fabsf(from) * -0x1p-21f ? 0.f : x;
                    }
                }
                dp[v] = groups.values(raw_up[v], v);
                if (a.drop.on) dp[v] = kept8(dp[v], dr, uint32_t(j) / 8u, uint32_t(row));
#pragma unroll
                for (int k = 0; k < 8; ++k) p[v][k] = exp_of<T>(p[v][k]);
                if (bits != 0xFFu) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        p[v][k] = bits >> k & 1u ? p[v][k] : 0.f;
                        dp[v][k] = bits >> k & 1u ? dp[v][k] : 0.f;
                    }
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) inner = fmaf(p[v][k], dp[v][k], inner);
            }
        }
        if constexpr (PHASE != WRITE) {
            inner = over_lanes<Add, LANES>(inner) * up_factor;
            if constexpr (TPR > 64) {   // this barrier also parts the rows' additions to the sums
                inner = over_waves<Add, TPR / 64>(inner, room[turn]);
                turn ^= 1u;
            }
        }
        if constexpr (PHASE == STATS) {
            if (t == 0u) a.part_stats[(row * a.row_parts + part) * 2u] = inner;
            continue;
        }
        if constexpr (PHASE == WRITE) {
            inner = 0.f;
            for (uint32_t q = 0; q < a.row_parts; ++q) inner += a.part_stats[(row * a.row_parts + q) * 2u];
            __syncthreads();
        }
        groups.store(o, [&](int v) {
            const int j = int(groups.col(v));
            f32x8 y = {};
            if (__any(j < r.limit)) {
                const uint32_t bits = admitted >> (8 * v) & 0xFFu;
#pragma unroll
                for (int k = 0; k < 8; ++k) p[v][k] *= fmaf(dp[v][k], up_factor, -inner);
                if (bits != 0xFFu) {   // a row's NaN stays where it looks
#pragma unroll
                    for (int k = 0; k < 8; ++k) p[v][k] = bits >> k & 1u ? p[v][k] : 0.f;
                }
                y = p[v] * a.scale;
                if (sums && bits) {
                    const Window w(r, j);
                    if (w.above(last) || w.below()) {
                        float e = 0.f;
#pragma unroll
                        for (int k = 0; k < 8; ++k) e += p[v][k];
                        low += w.below() ? e : 0.f;
                        high += w.below() ? 0.f : e;
                    } else {
                        // No two threads of a row have one distance, and a wave's accesses stay in order: read, add and write, which takes a tenth
                        // of the time of LDS atomics (75 cycles a wave), and gives the same sums every time.
                        volatile float *sum = acc;
                        float was[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) was[k] = sum[w.of(r, k)];
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[w.of(r, k)] = was[k] + p[v][k];
                    }
                }
            }
            return y;
        });
    }
    if constexpr (PHASE == STATS) return;
    if (!sums) return;
    low = over_lanes<Add, LANES>(low);
    high = over_lanes<Add, LANES>(high);
    __syncthreads();
    if constexpr (TPR > 64) {
        low = over_waves<Add, TPR / 64>(low, room[0]);
        high = over_waves<Add, TPR / 64>(high, room[1]);
    }
    if (t == 0u) {   // what lies beyond the ends is theirs
        for (uint32_t X = 0; X < kGuard; ++X) low += acc[cell(X)];
        for (uint32_t X = 1; X < kGuard; ++X) high += acc[cell(uint32_t(last) + kGuard + X)];
        acc[cell(kGuard)] += low;
        acc[cell(uint32_t(last) + kGuard)] += high;
    }
    __syncthreads();
    float *to = a.bias_sums + uint64_t(blockIdx.x) * (uint32_t(last) + 1u);
    for (uint32_t x = threadIdx.x; x <= uint32_t(last); x += WG) {
        float e = 0.f;
        for (uint32_t m = 0; m < TEAMS; ++m) e += lds[size * (1u + m) + cell(x + kGuard)];
        to[x] = e;
    }
}

// A workgroup to a head and bucket: its first wave lists the distances that have the bucket, and all add up what the backward pass's
// workgroups have for them, always in the same order.
__global__ __launch_bounds__(1024) void k_bias_reduce(BiasReduce a)
{
    extern __shared__ uint16_t mine[];   // [places]
    __shared__ float room[16];
    __shared__ uint32_t found_room;
    constexpr uint32_t AHEAD = 8;        // loads on their way
    const uint32_t n = a.places, h = blockIdx.x, bucket = blockIdx.y;
    if (threadIdx.x < 64u) {
        const uint32_t lane = threadIdx.x;
        uint32_t found = 0;
        for (uint32_t x0 = 0; x0 < n; x0 += 64u * AHEAD) {
            int32_t b[AHEAD];
#pragma unroll
            for (uint32_t u = 0; u < AHEAD; ++u) b[u] = x0 + u * 64u + lane < n ? min(max(a.map[x0 + u * 64u + lane], 0), int32_t(a.n_buckets) - 1) : -1;
#pragma unroll
            for (uint32_t u = 0; u < AHEAD; ++u) {
                const bool hit = b[u] == int32_t(bucket);
                const uint64_t hits = __ballot(hit);
                if (hit) mine[found + uint32_t(__popcll(hits & ((uint64_t(1) << lane) - 1u)))] = uint16_t(x0 + u * 64u + lane);
                found += uint32_t(__popcll(hits));
            }
        }
        if (lane == 0u) found_room = found;
    }
    __syncthreads();
    const uint32_t found = found_room, items = found * a.groups;   // below 4097 * 6 * 256
    const float *from = a.bias_sums + uint64_t(h) * a.groups * n;
    float e = 0.f;
    for (uint32_t i0 = threadIdx.x; i0 < items; i0 += 1024u * AHEAD) {
        float part[AHEAD];
#pragma unroll
        for (uint32_t u = 0; u < AHEAD; ++u) {
            const uint32_t i = min(i0 + u * 1024u, items - 1u), g = i / found;
            part[u] = from[uint64_t(g) * n + mine[i - g * found]];
        }
#pragma unroll
        for (uint32_t u = 0; u < AHEAD; ++u) e += i0 + u * 1024u < items ? part[u] : 0.f;
    }
    e = over_waves<Add, 16>(over_lanes<Add, 64>(e), room);
    if (threadIdx.x == 0u) {
        float *to = a.dtable + uint64_t(bucket) * a.heads + h;
        *to = a.accumulate ? *to + e : e;
    }
}

// ---- launches -----------------------------------------------------------------------------------------------------

static int check_launch() { return hipGetLastError() == hipSuccess ? ADACOMP_OK : ADACOMP_EHIP; }

constexpr uint32_t kPartThreads = 256, kPartGroups = 4, kPartKeys = kPartThreads * kPartGroups * 8u;
constexpr uint32_t kLdsMost = 40u << 10;      // of a workgroup: four of them fit a compute unit
constexpr uint32_t kMostWorkgroups = 1u << 20;   // of a launch, which has fewer than 2^32 threads; what is left is walked over

// Threads to a row and groups of 8 keys to a thread.  The LDS that the sums take is one bound, registers are another.  Few threads with up to 4 groups, since what a row costs whatever its length is then
// paid by few waves; in the backward pass, where a group takes twice the registers, 2 in short rows.  bf16, us, with 1 / 2 / 4 groups: forward
// 512 x 100 x 100 x 16 151 / 101 / 111, 256 x 200 x 200 x 16 240 / 201 / 147, 64 x 512 x 512 x 16 298 / 209 / 195, 4 x 512 x 6000 x 16 395 / 187 / 158;
// backward 202 / 154 / 305, 384 / 284 / 444, 509 / 376 / 400, 422 / 497 / 237.  Longer rows are cut into parts, and read twice.
SoftmaxForm softmax_form(uint32_t keys, uint32_t places, bool backward)
{
    if (backward) {   // every row that a workgroup has in hand has its sums by distance in LDS, beside the bias
        // and the rows get as many threads as leave room for that, with one group where it does: 64 x 16 x 600 x 250 with distances up to 800 and dropout
        // took 339 us in bf16 and 386 with two groups to a thread, 32 x 16 x 1500 x 400 691 and 730
        const uint32_t copies = kLdsMost / (4u * cells(places)) - 1u;
        if (copies < 16u && copies >= 8u && keys <= 256u) return {{32, 1}, 1};
        if (copies < 8u && copies >= 4u && keys <= 512u) return {{64, 1}, 1};
        keys = std::max(keys, copies >= 32u ? 0u : copies >= 16u ? 129u : copies >= 8u ? 257u : copies >= 4u ? 513u : 2049u);
    }
    if (keys <= 64u) return {{8, 1}, 1};
    if (keys <= 128u) return {{8, 2}, 1};
    if (keys <= 256u) return {{backward ? 16u : 8u, backward ? 2u : 4u}, 1};
    if (keys <= 512u) return {{backward ? 32u : 16u, backward ? 2u : 4u}, 1};
    if (keys <= 1024u) return {{backward ? 64u : 32u, backward ? 2u : 4u}, 1};
    if (keys <= 2048u) return {{64, 4}, 1};
    if (keys <= 4096u) return {{256, 2}, 1};
    if (keys <= 8192u) return {{256, 4}, 1};
    if (keys <= 16384u) return {{512, 4}, 1};
    if (keys <= 32768u) return {{1024, 4}, 1};
    return {{kPartThreads, kPartGroups}, (keys + kPartKeys - 1u) / kPartKeys};
}

// Workgroups of the backward pass to a head, with so many resident on a compute unit: as many as are resident in all, and no more, since
// those would wait for the others' ends (64 x 512 x 512 x 16 bf16 with 5 resident: 4, 5 and 6 to a unit take 375, 328 and 408 us).
static uint32_t back_groups(uint64_t rows_of_head, uint32_t heads, const SoftmaxForm &f, uint32_t resident)
{
    const uint64_t all = (rows_of_head * f.parts + f.row.teams() - 1u) / f.row.teams();
    const uint64_t most = std::max(1u, resident * kComputeUnits / heads), rounds = (all + most - 1u) / most;
    return rounds ? uint32_t((all + rounds - 1u) / rounds) : 0u;   // all with as many rows, up to one
}

uint32_t softmax_back_groups_most(uint64_t rows_of_head, uint32_t heads, const SoftmaxForm &f) { return back_groups(rows_of_head, heads, f, kMostResident); }

// Picks the kernel of a form and type and calls launch(kernel, phase) with it; twice where rows are cut into parts.
template <template <typename, int, int, int, int> class K, typename L>
static int with_kernel(const SoftmaxArgs &a, uint32_t dtype, const SoftmaxForm &f, L &&launch)
{
    constexpr bool BACK = K<float, 8, 1, WHOLE, PLAIN>::kBackward;
    const auto lines = [](const ViewArgs &v) { return (reinterpret_cast<uintptr_t>(v.data) | uint64_t(v.batch * 2) | uint64_t(v.head * 2) | uint64_t(v.row * 2)) % 64u == 0u; };
    // the backward pass, whose inputs are two thirds of its traffic: 320 us instead of 329; the forward pass gains nothing
    const bool once = BACK && !a.mask.data && dtype != ADACOMP_DTYPE_F32 && a.keys % 32u == 0u && lines(a.scores) && lines(a.in) &&
                      uint64_t(a.batch) * a.heads * a.queries * a.keys * 4u >= kInputsPast;
    auto go = [&](auto form, auto phase) {
        constexpr int TPR = decltype(form)::threads, V = decltype(form)::groups, PHASE = decltype(phase)::value;
        auto of = [&](auto kind) {
            constexpr int KIND = decltype(kind)::value;
            if constexpr (KIND != ONCE)
                if (dtype == ADACOMP_DTYPE_F32) return launch(std::integral_constant<void (*)(SoftmaxArgs), K<float, TPR, V, PHASE, KIND>::kernel>());
            if (dtype == ADACOMP_DTYPE_BF16) launch(std::integral_constant<void (*)(SoftmaxArgs), K<bf16, TPR, V, PHASE, KIND>::kernel>());
            else launch(std::integral_constant<void (*)(SoftmaxArgs), K<f16, TPR, V, PHASE, KIND>::kernel>());
        };
        if constexpr (BACK && PHASE == WHOLE && TPR > 8 && (V == 1 || (V == 2 && (TPR == 16 || TPR == 256))))   // what softmax_form gives to rows of fewer than 8 keys
            if (a.keys < 8u) return of(std::integral_constant<int, SHORT>());
        if constexpr (BACK && V * TPR >= 256 && PHASE == WHOLE)
            if (once) return of(std::integral_constant<int, ONCE>());
        if constexpr (!BACK && PHASE == WHOLE)
            if (a.merged) return a.mask.data ? of(std::integral_constant<int, MERGED_MASKED>()) : of(std::integral_constant<int, MERGED>());
        if (a.mask.data) of(std::integral_constant<int, MASKED>());
        else of(std::integral_constant<int, PLAIN>());
    };
    using Whole = std::integral_constant<int, WHOLE>;
    if (f.parts > 1u) {
        go(FormOf<kPartThreads, kPartGroups>(), std::integral_constant<int, STATS>());
        if (int rc = check_launch()) return rc;
        go(FormOf<kPartThreads, kPartGroups>(), std::integral_constant<int, WRITE>());
        return check_launch();
    }
    switch (f.row.threads * 8u + f.row.groups) {
    case 8 * 8 + 1: go(FormOf<8, 1>(), Whole()); break;
    case 8 * 8 + 2: go(FormOf<8, 2>(), Whole()); break;
    case 8 * 8 + 4: if constexpr (!BACK) go(FormOf<8, 4>(), Whole()); break;
    case 16 * 8 + 2: if constexpr (BACK) go(FormOf<16, 2>(), Whole()); break;
    case 16 * 8 + 4: if constexpr (!BACK) go(FormOf<16, 4>(), Whole()); break;
    case 32 * 8 + 1: if constexpr (BACK) go(FormOf<32, 1>(), Whole()); break;
    case 64 * 8 + 1: if constexpr (BACK) go(FormOf<64, 1>(), Whole()); break;
    case 32 * 8 + 2: if constexpr (BACK) go(FormOf<32, 2>(), Whole()); break;
    case 32 * 8 + 4: if constexpr (!BACK) go(FormOf<32, 4>(), Whole()); break;
    case 64 * 8 + 2: if constexpr (BACK) go(FormOf<64, 2>(), Whole()); break;
    case 64 * 8 + 4: go(FormOf<64, 4>(), Whole()); break;
    case 256 * 8 + 2: go(FormOf<256, 2>(), Whole()); break;
    case 256 * 8 + 4: go(FormOf<256, 4>(), Whole()); break;
    case 512 * 8 + 4: go(FormOf<512, 4>(), Whole()); break;
    case 1024 * 8 + 4: go(FormOf<1024, 4>(), Whole()); break;
    default: return ADACOMP_EINVAL;
    }
    return check_launch();
}

template <typename T, int TPR, int V, int PHASE, int KIND> struct KForward { static constexpr bool kBackward = false; static constexpr auto kernel = k_softmax_forward<T, TPR, V, PHASE, KIND>; };
template <typename T, int TPR, int V, int PHASE, int KIND> struct KBackward { static constexpr bool kBackward = true; static constexpr auto kernel = k_softmax_backward<T, TPR, V, PHASE, KIND>; };

// Shares the rows out to workgroups of the forward pass: to a team about 24000 keys, or 8 times what the bias takes to lay out, over the teams,
// and fewer where that leaves compute units without work.  Sequences of at most a quarter of a workgroup's rows share workgroups, head by head:
// 8000 x 16 x 17 x 17 in bf16 with dropout takes 160 us instead of 305, 4096 x 24 x 1 x 100 takes 18 instead of 148, 1024 x 16 x 60 x 60 takes 87 instead
// of 89, while 512 x 16 x 100 x 100, whose rows are nearly half of a workgroup's, would take 104 instead of 97.
static void share_rows(SoftmaxArgs &a, const SoftmaxForm &f)
{
    const uint32_t teams = f.row.teams(), wanted = std::max(24576u, 8u * a.places);
    uint32_t rows = std::min(std::max(wanted / (teams * std::max(a.keys, 1u)), teams == 1u ? 4u : 2u), 16u);
    for (;; --rows) {
        a.rows_per_wg = teams * rows;
        a.merged = a.batch > 1u && uint64_t(a.queries) * 4u <= a.rows_per_wg;
        const uint64_t together = a.merged ? uint64_t(a.batch) * a.queries : a.queries;
        a.wgs_per_head = uint32_t((together + a.rows_per_wg - 1u) / a.rows_per_wg);
        if (rows == 1u || uint64_t(a.merged ? 1u : a.batch) * a.heads * a.wgs_per_head >= 4u * kComputeUnits) return;
    }
}

int launch_softmax_forward(const SoftmaxArgs &args, uint32_t dtype, const SoftmaxForm &f, void *stream)
{
    SoftmaxArgs a = args;
    a.row_parts = f.parts;
    a.rows_per_wg = 1;
    a.wgs_per_head = a.queries;
    if (f.parts == 1u) share_rows(a, f);
    const uint64_t blocks = uint64_t(a.merged ? 1u : a.batch) * a.heads * a.wgs_per_head * f.parts;
    const dim3 grid(uint32_t(std::min<uint64_t>(blocks, kMostWorkgroups))), wg(f.row.workgroup());
    return with_kernel<KForward>(a, dtype, f, [&](auto kernel) {
        hipLaunchKernelGGL(kernel.value, grid, wg, 4u * cells(a.places), static_cast<hipStream_t>(stream), a);
    });
}

int launch_softmax_backward(const SoftmaxArgs &args, uint32_t dtype, const SoftmaxForm &f, uint32_t &groups, void *stream)
{
    SoftmaxArgs a = args;
    a.row_parts = f.parts;
    const uint32_t lds = 4u * cells(a.places) * (1u + (a.bias_sums ? f.row.teams() : 0u)), threads = f.row.workgroup();
    return with_kernel<KBackward>(a, dtype, f, [&](auto kernel) {
        // how many of the kernel's workgroups a compute unit holds with so much LDS: asked once, and again if the LDS differs
        static std::atomic<uint64_t> known{0};
        uint64_t k = known.load(std::memory_order_relaxed);
        if (k >> 32 != lds + 1u) {
            int n = 0;
            if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel.value, int(threads), lds) != hipSuccess) { (void)hipGetLastError(); n = 1; }
            k = uint64_t(lds + 1u) << 32 | uint32_t(std::min(std::max(n, 1), int(kMostResident)));
            known.store(k, std::memory_order_relaxed);
        }
        a.wgs_per_head = groups = back_groups(uint64_t(a.batch) * a.queries, a.heads, f, uint32_t(k));
        hipLaunchKernelGGL(kernel.value, dim3(a.heads * groups), dim3(threads), lds, static_cast<hipStream_t>(stream), a);
    });
}

int launch_bias_reduce(const BiasReduce &a, void *stream)
{
    const uint32_t lds = (2u * a.places + 15u) & ~15u;
    hipLaunchKernelGGL(k_bias_reduce, dim3(a.heads, a.n_buckets), dim3(1024), lds, static_cast<hipStream_t>(stream), a);
    return check_launch();
}

}  // namespace adacomp
