// sequence_recurrence.hip -- kernels of the gated linear recurrence (adacomp_sequence.h).
//
// A place changes the state by h -> m h + v, with v = (1 - a) x, and two such changes one after the other are one of the same kind:
// (m, v) then (m', v') is (m m', m' v + v').  So the threads of a workgroup share out a block of a sequence's places, each takes its own as
// one change, a scan over the threads says which state each of them begins with, and the block's last state is the next block's
// first.  The gradient goes the same way from the end: c -> m (c + d) at each place, with d = sigmoid(out) dy.
//
// A workgroup has a slab of 64 channels (a line of memory in 16 bits), 4 neighbouring ones to a thread, 16 threads beside each other, and
// walks along the sequence.  The 4 groups of 16 threads of a wave and the waves behind each other have runs of L places each.
//
// Forward reads x, forget and out and writes y, backward reads them and dy and writes their gradients.  8 x 2048 x 4096 bf16 with a gate: 123 us (4.4 TB/s),
// backward 220 (4.3 TB/s); without its exponentials the same kernel takes 123 and 218, so memory and its order bound it: rows of 128 bytes from 3 to 7 tensors (32 x
// 512 x 4096 126 us; 8 x 2048 x 2048, half of which the memory-side cache holds, 53 us, 5.0 TB/s).  Runs of 4 / 8 places in the forward pass of 16 bits 128 / 124
// us, and in the backward pass 227 / 617 (registers in memory).  With resets 132 and 232 us, for 15 % more vector instructions.  In parts, 1 x 65536 x 512
// f16 without a gate: 29 to 33 us for the changes and 38 to 40 for the walk (2.9 TB/s of what it needs, 4.9 of what it reads and writes).
#include "layers_device.h"
#include "sequence_plan.h"

namespace adacomp {

template <typename T> struct Raw4 { typedef T vec __attribute__((ext_vector_type(4))); typedef vec at __attribute__((aligned(sizeof(T)))); };
template <typename T> using raw4 = typename Raw4<T>::vec;
using f32x4 = raw4<float>;

// The 4 channels that a thread has, of which the last thread of a row may share some with its neighbour: it reads the row's last 4
// and writes those from `own` on.  Threads behind the row's end read its last 4 as well, and write none.  Where results share no memory with what is
// read they may write all 4: what they have for their neighbours' channels is what those write.
struct Channels {
    uint32_t first, own, count;   // count: channels read, 4 but in rows of fewer
    __device__ __forceinline__ Channels(uint32_t c, uint32_t channels)
    {
        count = min(channels, 4u);
        first = min(c, channels - count);
        own = c < channels ? c - first : 4u;
    }
    template <typename T> __device__ __forceinline__ raw4<T> load(const T *p) const   // p: at the row's channel `first`
    {
        if (count == 4u) return *reinterpret_cast<const typename Raw4<T>::at *>(p);
        raw4<T> v = {};
#pragma unroll
        for (uint32_t k = 0; k < 3u; ++k)
            if (k < count) v[k] = p[k];
        return v;
    }
    template <typename T> __device__ __forceinline__ void store(T *p, f32x4 x) const
    {
        const raw4<T> v = __builtin_convertvector(x, raw4<T>);
        if (own == 0u && count == 4u) { *reinterpret_cast<typename Raw4<T>::at *>(p) = v; return; }
#pragma unroll
        for (uint32_t k = 0; k < 4u; ++k)
            if (k >= own && k < count) p[k] = v[k];
    }
};

template <typename T> __device__ __forceinline__ f32x4 widen4(raw4<T> v) { return __builtin_convertvector(v, f32x4); }

// Values that the compiler takes for new ones: it would keep them widened across the scan otherwise, in twice the registers.
template <typename T, int L> __device__ __forceinline__ void renew(raw4<T> (&v)[L])
{
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(T))));
#pragma unroll
    for (int i = 0; i < L; ++i) {
        words w = __builtin_bit_cast(words, v[i]);
#pragma unroll
        for (uint32_t k = 0; k < sizeof(T); ++k) w[k] = again(w[k]);
        v[i] = __builtin_bit_cast(raw4<T>, w);
    }
}

// sigmoid(f) and sigmoid(-f), from e = exp(-|f|), which cannot leave the range: the smaller one is e / (1 + e), the larger one what is missing to 1.
// That difference is exact to half a step of the last place, where the reciprocal is not; a state that lasts for thousands of places
// has been multiplied by it as often.
struct Gate { float on, off; };
template <typename T> __device__ __forceinline__ Gate gate_of(float f)
{
    const float e = exp_of<T>(-fabsf(f)), small = e * __builtin_amdgcn_rcpf(1.f + e), big = 1.f - small;
    return {f > 0.f ? big : small, f > 0.f ? small : big};
}
// Where sigmoid(f) alone is wanted and only rounded.  exp(-f) may be an infinity: 1 / (1 + it) is 0.
template <typename T> __device__ __forceinline__ float sigmoid_of(float f)
{
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(f * -kLog2e));
    return gate_of<T>(f).on;
}

// A change of 4 channels' states.  With resets it says apart from m whether a document begins in it, and then nothing comes through, whatever m is: a product of
// gates may be NaN in front of the document, or too small for float32 without any.
template <bool RESETS> struct Change { f32x4 m, v; };
template <> struct Change<true> { f32x4 m, v; uint32_t cut; };

template <bool RESETS> __device__ __forceinline__ Change<RESETS> change_of(f32x4 m, f32x4 v, uint32_t cut)
{
    if constexpr (RESETS) return {m, v, cut};
    else return {m, v};
}
template <bool RESETS> __device__ __forceinline__ Change<RESETS> no_change() { return change_of<RESETS>(1.f, 0.f, 0u); }
template <bool RESETS> __device__ __forceinline__ uint32_t cut_of(const Change<RESETS> &c)
{
    if constexpr (RESETS) return c.cut;
    else return 0u;
}

template <bool RESETS> __device__ __forceinline__ f32x4 applied(const Change<RESETS> &c, f32x4 h)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        r[k] = fmaf(c.m[k], h[k], c.v[k]);
        if constexpr (RESETS) r[k] = c.cut ? c.v[k] : r[k];
    }
    return r;
}
// One change and then another.
template <bool RESETS> __device__ __forceinline__ Change<RESETS> then(const Change<RESETS> &one, const Change<RESETS> &other)
{
    return change_of<RESETS>(one.m * other.m, applied(other, one.v), cut_of(one) | cut_of(other));
}

// Backwards the gradient behind a place, with what the place adds, goes through it.
template <bool RESETS> __device__ __forceinline__ f32x4 back_through(const Change<RESETS> &c, f32x4 g) { return cut_of(c) ? f32x4(0.f) : c.m * g; }

// x of the even and the odd one of each two neighbouring groups of 16 lanes; of the lower and the upper half of the wave.
template <typename V> struct Two { V first, second; };
template <typename V> __device__ __forceinline__ Two<V> groups_of(V x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    return {__builtin_bit_cast(V, uint32_t(r[0])), __builtin_bit_cast(V, uint32_t(r[1]))};
}
template <typename V> __device__ __forceinline__ Two<V> halves_of(V x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return {__builtin_bit_cast(V, uint32_t(r[0])), __builtin_bit_cast(V, uint32_t(r[1]))};
}

// Over the 4 groups of 16 lanes of a wave, in their order or (BACK) from the last: what lies before each group, and `all` of them.
template <bool RESETS, bool BACK> __device__ __forceinline__ Change<RESETS> before_groups(const Change<RESETS> &own, Change<RESETS> &all)
{
    const uint32_t group = threadIdx.x % 64u / 16u;
    Change<RESETS> even, odd, lower, upper;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Two<float> m = groups_of(float(own.m[k])), v = groups_of(float(own.v[k]));
        even.m[k] = m.first; odd.m[k] = m.second;
        even.v[k] = v.first; odd.v[k] = v.second;
    }
    if constexpr (RESETS) {   // places are the same for the lanes of a group
        const Two<uint32_t> cut = groups_of(own.cut);
        even.cut = cut.first; odd.cut = cut.second;
    }
    const Change<RESETS> pair = BACK ? then(odd, even) : then(even, odd);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Two<float> m = halves_of(float(pair.m[k])), v = halves_of(float(pair.v[k]));
        lower.m[k] = m.first; upper.m[k] = m.second;
        lower.v[k] = v.first; upper.v[k] = v.second;
    }
    if constexpr (RESETS) {
        const Two<uint32_t> cut = halves_of(pair.cut);
        lower.cut = cut.first; upper.cut = cut.second;
    }
    all = BACK ? then(upper, lower) : then(lower, upper);
    Change<RESETS> before = no_change<RESETS>();
    if (BACK ? group < 2u : group >= 2u) before = BACK ? upper : lower;   // the other pair
    if (BACK ? group % 2u == 0u : group % 2u == 1u) before = then(before, BACK ? odd : even);   // the other one of the pair
    return before;
}

// The state that a thread begins with, in a workgroup that begins with `carry`, which becomes the one behind its last thread.
// room: of this block, and of every other one from then on.
template <int WAVES, bool RESETS, bool BACK>
__device__ __forceinline__ f32x4 begin_of(const Change<RESETS> &own, f32x4 &carry, Change<RESETS> (&room)[WAVES][16])
{
    const uint32_t lane = threadIdx.x % 64u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);
    Change<RESETS> all;
    const Change<RESETS> before = before_groups<RESETS, BACK>(own, all);
    if (lane < 16u) room[wave][lane] = all;
    __syncthreads();
    f32x4 mine = carry;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const int w = BACK ? WAVES - 1 - i : i;
        if (w == int(wave)) mine = carry;
        carry = applied(room[w][lane % 16u], carry);
    }
    return applied(before, mine);
}

// Which part of which sequence a workgroup has: slabs of a part are neighbours.
struct Job {
    uint32_t slab, segment, sequence, begin, end;   // places of the part
    __device__ __forceinline__ explicit Job(const RecurrenceArgs &a) : slab(blockIdx.x % a.slabs)
    {
        const uint32_t i = blockIdx.x / a.slabs;
        segment = i % a.segments;
        sequence = a.first_sequence + i / a.segments;
        begin = segment * a.segment;
        end = uint32_t(min(uint64_t(a.length), (segment + 1ull) * a.segment));
    }
};

// A tensor as a thread sees it.
struct Steps {
    const char *base;    // of the sequence; the same for a workgroup
    int64_t row;         // bytes
    uint32_t offset;     // of the thread from its wave's first place, where that is near
    template <typename T> __device__ __forceinline__ void set(const StepsArgs &s, uint32_t sequence, uint32_t places, uint32_t first)
    {
        base = static_cast<const char *>(s.data) + int64_t(sequence) * s.batch * int64_t(sizeof(T));
        row = s.row * int64_t(sizeof(T));
        offset = places * uint32_t(row) + first * uint32_t(sizeof(T));
    }
};

// What a thread has to do with: 4 channels and runs of L places.
template <typename T, int WAVES, int L> struct Place {
    static constexpr uint32_t kSteps = WAVES * 4u * L;   // places of a block
    Channels ch;
    uint32_t b, wave, run, length, end;   // run: first place inside a block; end: of the sequence
    bool whole;                           // every thread may read and write 4 channels, and rows are near each other
    f32x4 bias;
    __device__ __forceinline__ Place(const RecurrenceArgs &a, const Job &job)
        : ch(job.slab * kSlab + threadIdx.x % 16u * 4u, a.channels), b(job.sequence), wave(__builtin_amdgcn_readfirstlane(threadIdx.x / 64u)),
          run(threadIdx.x / 16u * L), length(a.length), end(a.length), whole(a.near_rows && ((job.slab + 1u) * kSlab <= a.channels || (a.apart && a.channels >= 4u)))
    {
        if (a.lengths) end = uint32_t(min(max(a.lengths[b], 0), int32_t(a.length)));
        bias = 0.f;
        if (a.bias) bias = ch.load(a.bias + ch.first);
    }
    __device__ __forceinline__ Steps steps(const StepsArgs &s) const
    {
        Steps r = {};
        if (s.data) r.template set<T>(s, b, threadIdx.x % 64u / 16u * L, ch.first);
        return r;
    }
    // Where the part's blocks without an exception end: every thread has L places and 4 channels there.
    __device__ __forceinline__ uint32_t full_end(const Job &job) const
    {
        const uint32_t upto = min(job.end, end);
        return whole && upto > job.begin ? job.begin + (upto - job.begin) / kSteps * kSteps : job.begin;
    }
    // Where the blocks with places inside the sequence end.
    __device__ __forceinline__ uint32_t live_end(const Job &job) const
    {
        const uint32_t upto = min(job.end, end);
        return upto > job.begin ? job.begin + (upto - job.begin + kSteps - 1u) / kSteps * kSteps : job.begin;
    }
    // Address of place i of the thread's run in a block.  FULL: an address that the wave shares, and a 32-bit offset.
    template <bool FULL> __device__ __forceinline__ T *at(const Steps &s, uint32_t block, int i) const
    {
        if constexpr (FULL) {
            const uintptr_t shared = reinterpret_cast<uintptr_t>(s.base) + uint64_t(int64_t(block + wave * 4u * L + i) * s.row);
            return reinterpret_cast<T *>(shared + s.offset);
        } else {
            const uint32_t t = min(block + run + i, length - 1u);
            return reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(s.base) + uint64_t(int64_t(t) * s.row) + ch.first * sizeof(T));
        }
    }
    // The thread's places; where there is none anything.
    template <bool FULL> __device__ __forceinline__ void load(raw4<T> (&to)[L], const Steps &s, uint32_t block) const
    {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if constexpr (FULL) to[i] = *reinterpret_cast<const typename Raw4<T>::at *>(at<FULL>(s, block, i));
            else to[i] = ch.load(static_cast<const T *>(at<FULL>(s, block, i)));
        }
    }
    template <bool FULL> __device__ __forceinline__ void load_resets(uint8_t (&to)[L], const RecurrenceArgs &a, uint32_t block) const
    {
        const uint8_t *row = a.resets + int64_t(b) * a.resets_stride;
#pragma unroll
        for (int i = 0; i < L; ++i) to[i] = row[FULL ? block + run + i : min(block + run + i, length - 1u)];
    }
    // Bit i: a document begins at place i of the run.
    template <bool FULL, bool RESETS> __device__ __forceinline__ uint32_t cuts_of(const uint8_t (&reset)[L], uint32_t block) const
    {
        uint32_t cuts = 0;
        if constexpr (RESETS)
#pragma unroll
            for (int i = 0; i < L; ++i) cuts |= reset[i] && inside<FULL>(block, i) ? 1u << i : 0u;
        return cuts;
    }
    template <bool FULL> __device__ __forceinline__ bool inside(uint32_t block, int i) const { return FULL || block + run + i < end; }
    // A value that counts only inside the sequence, whatever it is.
    template <bool FULL> __device__ __forceinline__ f32x4 value(raw4<T> raw, uint32_t block, int i) const { return inside<FULL>(block, i) ? widen4<T>(raw) : f32x4(0.f); }
    // a, 1 behind the end, and 1 - a of a place
    template <bool FULL> __device__ __forceinline__ void gates(raw4<T> forget, uint32_t block, int i, f32x4 &a, f32x4 &rest) const
    {
        const f32x4 f = widen4<T>(forget) + bias;
        const bool in = inside<FULL>(block, i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const Gate g = gate_of<T>(f[k]);
            a[k] = in ? g.on : 1.f;
            rest[k] = in ? g.off : 0.f;
        }
    }
    // Results go past the caches. 8 x 2048 x 2000 bf16: forward 69.0 us (through them 70.3), backward 153 to 162 (169); rows that begin at odd addresses, 2001
    // channels: forward 84.5 (85.3), but backward 203 to 209 (186). A branch that chose cost the aligned rows more (178) than it gave the odd ones (197).
    template <bool FULL> __device__ __forceinline__ void store(const Steps &s, uint32_t block, int i, f32x4 x) const
    {
        if constexpr (FULL) __builtin_nontemporal_store(__builtin_convertvector(x, raw4<T>), reinterpret_cast<typename Raw4<T>::at *>(at<FULL>(s, block, i)));
        else if (block + run + i < length) ch.store(at<FULL>(s, block, i), inside<FULL>(block, i) ? x : f32x4(0.f));
    }
    __device__ __forceinline__ uint64_t state(uint32_t channels, uint64_t i) const { return i * channels + ch.first; }
};

// ---- sequences in several parts -----------------------------------------------------------------------------------
// Few sequences of few channels are cut into parts.  One launch says what each part does to the state (BACK: to the gradient that comes from
// behind), as one change; the next one's workgroups put the changes before their part together and walk along it.  Here nothing
// but the end of a part is wanted, so each group of 16 threads goes along a run of its own, without a scan until the last place.
// With resets m is -0 where a document begins in the part: gates and their products are never negative.
// The part that nobody comes behind has the place of its change for the state that the sequence begins with: the second launch does not read that where
// the caller has it, since the last state may be written over it.

template <typename T, int WAVES, int L, bool RESETS, bool BACK, bool GATE> __global__ __launch_bounds__(WAVES * 64) void k_recurrence_changes(RecurrenceArgs a)
{
    __shared__ Change<RESETS> room[WAVES][16];
    const Job job(a);
    const Place<T, WAVES, L> p(a, job);
    float *to = a.changes + (uint64_t(job.sequence) * a.segments + job.segment) * 2u * a.channels + p.ch.first;
    if (job.segment == (BACK ? 0u : a.segments - 1u)) {
        if (threadIdx.x < 16u) p.ch.store(to, a.first ? p.ch.load(a.first + p.state(a.channels, p.b)) : f32x4(0.f));
        return;
    }
    const uint32_t last = max(min(job.end, p.end), job.begin);   // places behind the sequence's end change nothing
    const uint32_t each = (last - job.begin + WAVES * 4u - 1u) / (WAVES * 4u), group = threadIdx.x / 16u;
    const uint32_t begin = min(job.begin + group * each, last), count = min(each, last - begin);
    const Steps forget_of = p.steps(a.forget), other_of = p.steps(BACK ? a.y : a.x), out_of = p.steps(a.out);
    const uint8_t *resets = RESETS ? a.resets + int64_t(p.b) * a.resets_stride : nullptr;
    Change<RESETS> all = no_change<RESETS>();
    for (uint32_t n = 0; n < count; n += L) {
        raw4<T> forget[L], other[L], out[L];
        uint8_t reset[L];
        // place i, or the nearest one that is there
        auto place = [&](int i) { const uint32_t k = min(n + i, count - 1u); return BACK ? begin + count - 1u - k : begin + k; };
        auto inside = [&](int i) { return n + i < count; };
        auto load = [&](raw4<T> (&to)[L], const Steps &s) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < L; ++i) to[i] = p.ch.load(reinterpret_cast<const T *>(s.base + int64_t(place(i)) * s.row + p.ch.first * sizeof(T)));
        };
        load(forget, forget_of);
        load(other, other_of);
        if constexpr (BACK && GATE) load(out, out_of);
        if constexpr (RESETS)
#pragma unroll
            for (int i = 0; i < L; ++i) reset[i] = resets[place(i)];
#pragma unroll
        for (int i = 0; i < L; ++i) {
            const bool in = inside(i);
            const f32x4 f = widen4<T>(forget[i]) + p.bias;
            f32x4 v = widen4<T>(other[i]);
            if constexpr (BACK && GATE) {
                const f32x4 o = widen4<T>(out[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] *= sigmoid_of<T>(o[k]);
            }
            Change<RESETS> c = no_change<RESETS>();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const Gate g = gate_of<T>(f[k]);
                c.m[k] = in ? g.on : 1.f;
                c.v[k] = !in ? 0.f : BACK ? v[k] : g.off * v[k];
            }
            if constexpr (RESETS) c.cut = in && reset[i];
            if constexpr (BACK) {   // what comes from behind and what the place adds go through it together
                c.v = back_through(c, c.v + all.v);
                all = change_of<RESETS>(all.m * c.m, c.v, cut_of(all) | cut_of(c));
            } else {
                all = then(all, c);
            }
        }
    }
    // the change of the whole part: what the groups do one after the other
    Change<RESETS> of_wave;
    before_groups<RESETS, BACK>(all, of_wave);
    const uint32_t lane = threadIdx.x % 64u;
    if (lane < 16u) room[threadIdx.x / 64u][lane] = of_wave;
    __syncthreads();
    if (threadIdx.x >= 16u) return;
    Change<RESETS> total = no_change<RESETS>();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) total = then(total, room[BACK ? WAVES - 1 - i : i][lane]);
    p.ch.store(to, cut_of(total) ? f32x4(-0.f) : total.m);
    p.ch.store(to + a.channels, total.v);
}

// The state that a part begins with (BACK: the gradient from behind it), from that of the sequence: groups of 16 threads put runs of the
// changes before it together.
template <int WAVES, bool RESETS, bool BACK, typename P>
__device__ __forceinline__ f32x4 begin_of_part(const RecurrenceArgs &a, const P &p, const Job &job, Change<RESETS> (&room)[WAVES][16])
{
    f32x4 carry = 0.f;
    if (a.segments == 1u) {
        if (a.first) carry = p.ch.load(a.first + p.state(a.channels, p.b));
        return carry;
    }
    carry = p.ch.load(a.changes + (uint64_t(job.sequence) * a.segments + (BACK ? 0u : a.segments - 1u)) * 2u * a.channels + p.ch.first);
    const uint32_t before = BACK ? a.segments - 1u - job.segment : job.segment, each = (before + WAVES * 4u - 1u) / (WAVES * 4u), group = threadIdx.x / 16u;
    const uint32_t order = BACK ? WAVES * 4u - 1u - group : group;
    Change<RESETS> all = no_change<RESETS>();
    for (uint32_t i = order * each; i < min((order + 1u) * each, before); ++i) {
        const uint32_t segment = BACK ? a.segments - 1u - i : i;
        const float *from = a.changes + (uint64_t(job.sequence) * a.segments + segment) * 2u * a.channels + p.ch.first;
        const f32x4 m = p.ch.load(from);
        all = then(all, change_of<RESETS>(m, p.ch.load(from + a.channels), __builtin_bit_cast(uint32_t, float(m[0])) == 0x80000000u));
    }
    begin_of<WAVES, RESETS, BACK>(all, carry, room);
    return carry;
}

// ---- the walk along a sequence or a part of it --------------------------------------------------------------------
// Blocks without an exception have a loop of their own, in which the next block's values are on their way while a block is worked on: no branch
// stands between its loads and stores, or the wait for the loads would be one for the stores behind them too.

template <typename T, int WAVES, int L, bool RESETS, bool GATE> __global__ __launch_bounds__(WAVES * 64, 2) void k_recurrence_forward(RecurrenceArgs a)
{
    using P = Place<T, WAVES, L>;
    __shared__ Change<RESETS> room[3][WAVES][16];
    const Job job(a);
    const P p(a, job);
    const Steps x_of = p.steps(a.x), forget_of = p.steps(a.forget), out_of = p.steps(a.out), y_of = p.steps(a.y);
    raw4<T> x[L], forget[L], out[L] = {};
    uint8_t reset[L] = {};
    auto fetch = [&](uint32_t block, auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        p.template load<FULL>(x, x_of, block);
        p.template load<FULL>(forget, forget_of, block);
        if constexpr (GATE) p.template load<FULL>(out, out_of, block);
        if constexpr (RESETS) p.template load_resets<FULL>(reset, a, block);
    };
    const uint32_t full_end = p.full_end(job), live_end = p.live_end(job);   // blocks before them are full, or have places inside the sequence
    if (job.begin < full_end) fetch(job.begin, std::true_type());
    f32x4 carry = begin_of_part<WAVES, RESETS, false>(a, p, job, room[2]);
    uint32_t turn = 0;
    auto keep = [&](uint32_t t, f32x4 h) __attribute__((always_inline)) {
        if (a.states && t % ADACOMP_RECURRENCE_KEEP == 0u && t < a.length) p.ch.store(a.states + p.state(a.channels, uint64_t(p.b) * a.kept + t / ADACOMP_RECURRENCE_KEEP), h);
    };
    auto work = [&](uint32_t block, auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        raw4<T> out_now[L];
        f32x4 m[L], v[L];
        Change<RESETS> all = no_change<RESETS>();
        if constexpr (!FULL) fetch(block, full);
        const uint32_t cuts = p.template cuts_of<FULL, RESETS>(reset, block);
        auto step = [&](int i) __attribute__((always_inline)) { return change_of<RESETS>(m[i], v[i], cuts & 1u << i); };
#pragma unroll
        for (int i = 0; i < L; ++i) {
            f32x4 rest;
            p.template gates<FULL>(forget[i], block, i, m[i], rest);
            v[i] = rest * p.template value<FULL>(x[i], block, i);
            all = then(all, step(i));
            out_now[i] = out[i];
        }
        if constexpr (FULL) fetch(min(block + P::kSteps, full_end - P::kSteps), full);
        f32x4 h = begin_of<WAVES, RESETS, false>(all, carry, room[turn]);
        turn ^= 1u;
        renew<T>(out_now);
        const uint32_t t0 = block + p.run;
        keep(t0, h);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            h = applied(step(i), h);
            f32x4 y = h;
            if constexpr (GATE) {
                const f32x4 o = widen4<T>(out_now[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] *= sigmoid_of<T>(o[k]);
            }
            p.template store<FULL>(y_of, block, i, y);
        }
    };
    for (uint32_t block = job.begin; block < full_end; block += P::kSteps) work(block, std::true_type());
    for (uint32_t block = full_end; block < live_end; block += P::kSteps) work(block, std::false_type());
    for (uint32_t block = live_end; block < job.end; block += P::kSteps) {
        keep(block + p.run, carry);
        for (int i = 0; i < L; ++i) p.template store<false>(y_of, block, i, f32x4(0.f));
    }
    if (a.last && job.segment + 1u == a.segments && threadIdx.x < 16u) p.ch.store(a.last + p.state(a.channels, p.b), carry);
}

template <typename T, int WAVES, int L, bool RESETS, bool GATE> __global__ __launch_bounds__(WAVES * 64, 2) void k_recurrence_backward(RecurrenceArgs a)
{
    using P = Place<T, WAVES, L>;
    static_assert(ADACOMP_RECURRENCE_KEEP % P::kSteps == 0 || P::kSteps % ADACOMP_RECURRENCE_KEEP == 0, "a block begins with a state that was kept, or is the only one");
    __shared__ Change<RESETS> room[5][WAVES][16];
    __shared__ f32x4 sums[WAVES * 4][16];
    const Job job(a);
    const P p(a, job);
    const Steps x_of = p.steps(a.x), forget_of = p.steps(a.forget), out_of = p.steps(a.out), dy_of = p.steps(a.y), dx_of = p.steps(a.dx), df_of = p.steps(a.dforget),
                dout_of = p.steps(a.dout);
    raw4<T> next_x[L], next_forget[L], next_out[L] = {}, next_dy[L];
    uint8_t next_reset[L] = {};
    f32x4 next_state;
    auto fetch = [&](uint32_t block, auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        p.template load<FULL>(next_x, x_of, block);
        p.template load<FULL>(next_forget, forget_of, block);
        p.template load<FULL>(next_dy, dy_of, block);
        if constexpr (GATE) p.template load<FULL>(next_out, out_of, block);
        if constexpr (RESETS) p.template load_resets<FULL>(next_reset, a, block);
        next_state = p.ch.load(a.states + p.state(a.channels, uint64_t(p.b) * a.kept + block / ADACOMP_RECURRENCE_KEEP));
    };
    const uint32_t full_end = p.full_end(job), live_end = p.live_end(job);
    f32x4 carry = begin_of_part<WAVES, RESETS, true>(a, p, job, room[4]), dbias = 0.f;
    uint32_t turn = 0;
    auto work = [&](uint32_t block, auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
        if constexpr (!FULL) fetch(block, full);
        raw4<T> x[L], out[L], dy[L];
        f32x4 m[L], rest[L], state = next_state;   // m: a
        Change<RESETS> all = no_change<RESETS>(), back = all;
        const uint32_t cuts = p.template cuts_of<FULL, RESETS>(next_reset, block);
        auto step = [&](int i) __attribute__((always_inline)) { return change_of<RESETS>(m[i], rest[i] * p.template value<FULL>(x[i], block, i), cuts & 1u << i); };
#pragma unroll
        for (int i = 0; i < L; ++i) {
            x[i] = next_x[i];
            out[i] = next_out[i];
            dy[i] = next_dy[i];
            p.template gates<FULL>(next_forget[i], block, i, m[i], rest[i]);
            all = then(all, step(i));
        }
        if constexpr (FULL) fetch(max(block, job.begin + P::kSteps) - P::kSteps, full);
#pragma unroll
        for (int i = L - 1; i >= 0; --i) {
            f32x4 d = p.template value<FULL>(dy[i], block, i);
            if constexpr (GATE) {
                const f32x4 o = p.template value<FULL>(out[i], block, i);
#pragma unroll
                for (int k = 0; k < 4; ++k) d[k] *= sigmoid_of<T>(o[k]);
            }
            back.v = back_through(step(i), d + back.v);
        }
        back = change_of<RESETS>(all.m, back.v, cut_of(all));
        f32x4 h[L];   // before each place
        h[0] = begin_of<WAVES, RESETS, false>(all, state, room[turn * 2u]);
        f32x4 c = begin_of<WAVES, RESETS, true>(back, carry, room[turn * 2u + 1u]);
        turn ^= 1u;
        renew<T>(x);
        renew<T>(out);
        renew<T>(dy);
#pragma unroll
        for (int i = 1; i < L; ++i) h[i] = applied(step(i - 1), h[i - 1]);
#pragma unroll
        for (int i = L - 1; i >= 0; --i) {
            const f32x4 xi = p.template value<FULL>(x[i], block, i), up = p.template value<FULL>(dy[i], block, i);
            const f32x4 came = cut_of(step(i)) ? f32x4(0.f) : h[i];
            f32x4 g = up, df, dout;
            if constexpr (GATE) {
                const f32x4 o = p.template value<FULL>(out[i], block, i);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const Gate gate = gate_of<T>(o[k]);
                    g[k] *= gate.on;
                    dout[k] = up[k] * fmaf(m[i][k], came[k], rest[i][k] * xi[k]) * (gate.on * gate.off);
                }
                p.template store<FULL>(dout_of, block, i, dout);
            }
            g += c;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                c[k] = cut_of(step(i)) ? 0.f : m[i][k] * g[k];
                df[k] = g[k] * (m[i][k] * rest[i][k]) * (came[k] - xi[k]);   // behind the end `rest` is 0
            }
            if (!p.template inside<FULL>(block, i)) df = 0.f;
            dbias += df;
            p.template store<FULL>(dx_of, block, i, g * rest[i]);
            p.template store<FULL>(df_of, block, i, df);
        }
    };
    for (uint32_t block = live_end; block < job.end; block += P::kSteps)
        for (int i = 0; i < L; ++i) {
            p.template store<false>(dx_of, block, i, f32x4(0.f));
            p.template store<false>(df_of, block, i, f32x4(0.f));
            if constexpr (GATE) p.template store<false>(dout_of, block, i, f32x4(0.f));
        }
    for (uint32_t n = (live_end - full_end) / P::kSteps; n-- > 0u;) work(full_end + n * P::kSteps, std::false_type());
    if (full_end > job.begin) {
        fetch(full_end - P::kSteps, std::true_type());
        for (uint32_t n = (full_end - job.begin) / P::kSteps; n-- > 0u;) work(job.begin + n * P::kSteps, std::true_type());
    }
    if (a.last && job.segment == 0u && threadIdx.x < 16u) p.ch.store(a.last + p.state(a.channels, p.b), carry);
    if (!a.dbias_parts) return;
    sums[threadIdx.x / 16u][threadIdx.x % 16u] = dbias;
    __syncthreads();
    if (threadIdx.x >= 16u) return;
    f32x4 s = 0.f;
    for (uint32_t g = 0; g < WAVES * 4u; ++g) s += sums[g][threadIdx.x];
    p.ch.store(a.dbias_parts + p.state(a.channels, uint64_t(p.b) * a.segments + job.segment), s);
}

// Sequences of few places, single tokens above all, and calls of so many sequences and channels that every one can have a thread: it takes 4
// channels of a sequence from the first place to the last.
template <typename T, int L, bool RESETS, bool GATE> __global__ __launch_bounds__(256) void k_recurrence_few(RecurrenceArgs a)
{
    const uint32_t groups = (a.channels + 3u) / 4u, i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t b = a.first_sequence + i / groups;
    if (b >= a.batch) return;
    const Channels ch(i % groups * 4u, a.channels);
    const uint64_t state = uint64_t(b) * a.channels + ch.first;
    auto address = [&](const StepsArgs &s, uint32_t t) __attribute__((always_inline)) {
        return static_cast<T *>(const_cast<void *>(s.data)) + int64_t(b) * s.batch + int64_t(t) * s.row + ch.first;
    };
    f32x4 bias = 0.f, h = 0.f;
    if (a.bias) bias = ch.load(a.bias + ch.first);
    if (a.first) h = ch.load(a.first + state);
    uint32_t end = a.length;
    if (a.lengths) end = uint32_t(min(max(a.lengths[b], 0), int32_t(a.length)));
    for (uint32_t t = 0; t < a.length; t += L) {
        raw4<T> x[L], forget[L], out[L];
        uint8_t reset[L] = {};
#pragma unroll
        for (int k = 0; k < L; ++k) {
            const uint32_t at = min(t + k, a.length - 1u);
            x[k] = ch.load(address(a.x, at));
            forget[k] = ch.load(address(a.forget, at));
            if constexpr (GATE) out[k] = ch.load(address(a.out, at));
            if constexpr (RESETS) reset[k] = a.resets[int64_t(b) * a.resets_stride + at];
        }
#pragma unroll
        for (int k = 0; k < L; ++k) {
            if (t + k >= a.length) break;
            if (a.states && (t + k) % ADACOMP_RECURRENCE_KEEP == 0u) ch.store(a.states + (uint64_t(b) * a.kept + (t + k) / ADACOMP_RECURRENCE_KEEP) * a.channels + ch.first, h);
            const f32x4 f = widen4<T>(forget[k]) + bias, xk = widen4<T>(x[k]);
            f32x4 y = 0.f;
            if (t + k < end) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const Gate g = gate_of<T>(f[c]);
                    h[c] = fmaf(g.off, xk[c], RESETS && reset[k] ? 0.f : g.on * h[c]);
                    y[c] = h[c];
                    if constexpr (GATE) y[c] *= sigmoid_of<T>(float(out[k][c]));
                }
            }
            ch.store(address(a.y, t + k), y);
        }
    }
    if (a.last) ch.store(a.last + state, h);
}

// dbias[c] = sum over the parts, in their order.  32 channels to a workgroup, 32 slices of the parts.
__global__ __launch_bounds__(1024) void k_bias_sum(BiasSumArgs a)
{
    __shared__ float sums[32][33];
    const uint32_t lane = threadIdx.x % 32u, slice = threadIdx.x / 32u, c = blockIdx.x * 32u + lane;
    float s = 0.f;
    if (c < a.channels)
        for (uint32_t p = slice; p < a.count; p += 32u) s += a.parts[uint64_t(p) * a.channels + c];
    sums[slice][lane] = s;
    __syncthreads();
    if (slice != 0u || c >= a.channels) return;
    float all = 0.f;
    for (uint32_t k = 0; k < 32u; ++k) all += sums[k][lane];
    a.dbias[c] = a.accumulate ? a.dbias[c] + all : all;
}

// ---- launches -----------------------------------------------------------------------------------------------------

constexpr int kWaves = 4;
template <typename T> constexpr int kForwardRun = sizeof(T) == 2 ? 8 : 4;
// The backward pass of 32-bit tensors with a gate has registers for half as many places (8 x 2048 x 2048 308 / 212 us, 47 to 123 registers in memory
// otherwise; without a gate 152 / 156).
template <typename T, bool GATE> constexpr int kBackwardRun = sizeof(T) == 4 && GATE ? 2 : 4;

// Whether a call goes place by place: one place after the other takes 0.6 us, a workgroup's block of them 14 ns and a call of few of those 9 us
// (512 x 16 x 4096 bf16 48 / 453 us, 512 x 64 x 4096 229 / 479, 256 x 64 x 1024 40 / 56, 32 x 32 x 4096 22 / 29, 32 x 48 x 4096 31 / 30, 4 x 8 x 512 9 / 9,
// 4 x 16 x 512 10.8 / 9.0).
static bool place_by_place(const RecurrenceArgs &a) { return a.length <= std::max<uint64_t>(12u, uint64_t(a.batch) * a.slabs / 48u); }

// Calls f with the arguments and the grid of every launch.
template <typename F> static int for_sequences(const RecurrenceArgs &args, F &&f)
{
    RecurrenceArgs a = args;
    const uint32_t of_one = a.slabs * a.segments, step = recurrence_sequences(of_one);
    for (uint64_t first = 0; first < args.batch; first += step) {
        a.first_sequence = uint32_t(first);
        if (int rc = f(a, dim3(uint32_t(std::min<uint64_t>(step, args.batch - first)) * of_one))) return rc;
    }
    return ADACOMP_OK;
}

template <typename F> static int with_form(const RecurrenceArgs &a, uint32_t dtype, F &&f)
{
    return with_type(dtype, [&](auto of) {
        const auto gate = [&](auto resets) {
            if (a.out.data) f(of, resets, std::true_type());
            else f(of, resets, std::false_type());
        };
        if (a.resets) gate(std::true_type());
        else gate(std::false_type());
    });
}

int launch_recurrence_forward(const RecurrenceArgs &args, uint32_t dtype, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (place_by_place(args)) {
        RecurrenceArgs a = args;
        const uint32_t groups = (a.channels + 3u) / 4u, step = (1u << 30) / groups;   // threads of a launch are counted in 32 bits
        for (uint64_t first = 0; first < args.batch; first += step) {
            a.first_sequence = uint32_t(first);
            a.batch = uint32_t(std::min<uint64_t>(args.batch, first + step));
            const dim3 grid(((a.batch - a.first_sequence) * groups + 255u) / 256u);
            const int rc = with_form(a, dtype, [&](auto of, auto resets, auto gate) {
                using T = decltype(of);
                constexpr bool RESETS = decltype(resets)::value, GATE = decltype(gate)::value;
                if (a.length <= 2u) hipLaunchKernelGGL((k_recurrence_few<T, 1, RESETS, GATE>), grid, dim3(256), 0, s, a);
                else hipLaunchKernelGGL((k_recurrence_few<T, 4, RESETS, GATE>), grid, dim3(256), 0, s, a);
            });
            if (rc) return rc;
        }
        return ADACOMP_OK;
    }
    return for_sequences(args, [&](const RecurrenceArgs &a, dim3 grid) {
        return with_form(a, dtype, [&](auto of, auto resets, auto gate) {
            using T = decltype(of);
            constexpr bool RESETS = decltype(resets)::value, GATE = decltype(gate)::value;
            static_assert(kWaves * 64u <= kRecurrenceThreads);
            if (a.segments > 1u) hipLaunchKernelGGL((k_recurrence_changes<T, 4, 8, RESETS, false, false>), grid, dim3(256), 0, s, a);
            hipLaunchKernelGGL((k_recurrence_forward<T, kWaves, kForwardRun<T>, RESETS, GATE>), grid, dim3(kWaves * 64), 0, s, a);
        });
    });
}

int launch_recurrence_backward(const RecurrenceArgs &args, uint32_t dtype, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    return for_sequences(args, [&](const RecurrenceArgs &a, dim3 grid) {
        return with_form(a, dtype, [&](auto of, auto resets, auto gate) {
            using T = decltype(of);
            constexpr bool RESETS = decltype(resets)::value, GATE = decltype(gate)::value;
            if (a.segments > 1u) hipLaunchKernelGGL((k_recurrence_changes<T, 4, 8, RESETS, true, GATE>), grid, dim3(256), 0, s, a);
            constexpr int L = kBackwardRun<T, GATE>, WAVES = 16 / L;   // blocks of 64 places, or 16 or 32 where the sequence has no more
            static_assert(WAVES * 64u <= kRecurrenceThreads);
            if (a.length <= 16u) hipLaunchKernelGGL((k_recurrence_backward<T, WAVES / 4, L, RESETS, GATE>), grid, dim3(WAVES * 16), 0, s, a);
            else if (a.length <= 32u) hipLaunchKernelGGL((k_recurrence_backward<T, WAVES / 2, L, RESETS, GATE>), grid, dim3(WAVES * 32), 0, s, a);
            else hipLaunchKernelGGL((k_recurrence_backward<T, WAVES, L, RESETS, GATE>), grid, dim3(WAVES * 64), 0, s, a);
        });
    });
}

int launch_bias_sum(const BiasSumArgs &a, void *stream)
{
    hipLaunchKernelGGL(k_bias_sum, dim3((a.channels + 31u) / 32u), dim3(1024), 0, static_cast<hipStream_t>(stream), a);
    return check_launch();
}

}  // namespace adacomp
