// sequence_recurrence.hip -- kernels of the gated linear recurrence (adacomp_sequence.h).
//
// A place changes the state by h -> m h + v, with v = (1 - a) x, and two such changes one after the other are one of the same kind:
// (m, v) then (m', v') is (m m', m' v + v').  So the threads of a workgroup share out a block of a sequence's places, each takes its own as
// one change, a scan over the threads says which state each of them begins with, and the block's last state is the next block's
// first.  The gradient goes the same way from the end: c -> m (c + d) at each place, with d = sigmoid(out) dy.
//
// A workgroup has a slab of 64 channels (a line of memory in 16 bits), 4 neighbouring ones to a thread, 16 threads beside each other, and
// walks along the sequence.  The 4 groups of 16 threads of a wave and the waves behind each other have runs of L places each.
#include "layers_device.h"
#include "sequence_plan.h"

namespace adacomp {

template <typename T> struct Raw4 { typedef T vec __attribute__((ext_vector_type(4))); typedef vec at __attribute__((aligned(sizeof(T)))); };
template <typename T> using raw4 = typename Raw4<T>::vec;
using f32x4 = raw4<float>;

// The 4 channels that a thread has, of which the last thread of a row may share some with its neighbour: it reads the row's last 4
// and writes those from `own` on.
struct Channels {
    uint32_t first, own, count;   // count: channels read, 4 but in rows of fewer
    bool live;
    __device__ __forceinline__ Channels(uint32_t c, uint32_t channels)
    {
        live = c < channels;
        count = min(channels, 4u);
        first = min(c, channels - count);
        own = live ? c - first : 4u;
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

struct Gate { float on, off; };   // sigmoid(f), sigmoid(-f)

// 1 - sigmoid as a value of its own: near 1 the difference would have lost its digits.  Below -80 exp(-f) would leave the range.
template <typename T> __device__ __forceinline__ Gate gate_of(float f)
{
    const float e = exp_of<T>(-(f < -80.f ? -80.f : f)), on = __builtin_amdgcn_rcpf(1.f + e);
    return {on, e * on};
}

// The gate of the state, whose error is multiplied over as many places as the state lasts: the exponential that float32 tensors have, and near 1,
// where it lasts long, the sigmoid from the exact difference.
__device__ __forceinline__ Gate state_gate_of(float f)
{
    const Gate g = gate_of<float>(f);
    return {f > 0.f ? 1.f - g.off : g.on, g.off};
}

// What comes through a place: nothing through one that begins a document, whatever it is.
template <bool RESETS> __device__ __forceinline__ float through(float m, float h)
{
    if constexpr (RESETS) return m == 0.f ? 0.f : m * h;
    return m * h;
}

// A change of 4 channels' states.
struct Change { f32x4 m, v; };

template <bool RESETS> __device__ __forceinline__ f32x4 applied(const Change &c, f32x4 h)
{
    f32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = RESETS ? through<RESETS>(c.m[k], h[k]) + c.v[k] : fmaf(c.m[k], h[k], c.v[k]);
    return r;
}

// Over the 4 groups of 16 lanes of a wave, in their order or (BACK) from the last: what lies before each group, and `all`, valid in the
// last one (BACK: the first).
template <bool RESETS, bool BACK> __device__ __forceinline__ Change before_groups(const Change &own, Change &all)
{
    const uint32_t group = threadIdx.x % 64u / 16u, order = BACK ? 3u - group : group;
    auto from = [](float x, uint32_t by) { return BACK ? __shfl_down(x, by) : __shfl_up(x, by); };
    Change c = own;
#pragma unroll
    for (uint32_t step = 1; step < 4u; step *= 2u) {
        Change other;
#pragma unroll
        for (int k = 0; k < 4; ++k) { other.m[k] = from(c.m[k], 16u * step); other.v[k] = from(c.v[k], 16u * step); }
        if (order >= step) {
            c.v = applied<RESETS>(c, other.v);
            c.m *= other.m;
        }
    }
    all = c;
    Change before;
#pragma unroll
    for (int k = 0; k < 4; ++k) { before.m[k] = from(c.m[k], 16u); before.v[k] = from(c.v[k], 16u); }
    if (order == 0u) { before.m = 1.f; before.v = 0.f; }
    return before;
}

// The state that a thread begins with, in a workgroup that begins with `carry`, which becomes the one behind its last thread.
// room: of this block, and of every other one from then on.
template <int WAVES, bool RESETS, bool BACK>
__device__ __forceinline__ f32x4 begin_of(const Change &own, f32x4 &carry, Change (&room)[WAVES][16])
{
    const uint32_t lane = threadIdx.x % 64u, wave = threadIdx.x / 64u;
    Change all;
    const Change before = before_groups<RESETS, BACK>(own, all);
    if (lane / 16u == (BACK ? 0u : 3u)) room[wave][lane % 16u] = all;
    __syncthreads();
    f32x4 mine = carry;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        const int w = BACK ? WAVES - 1 - i : i;
        if (w == int(wave)) mine = carry;
        carry = applied<RESETS>(room[w][lane % 16u], carry);
    }
    return applied<RESETS>(before, mine);
}

// What a thread has to do with.
template <typename T, int WAVES, int L> struct Place {
    static constexpr uint32_t kSteps = WAVES * 4u * L;   // places of a block
    Channels ch;
    uint32_t b, run, length, end;   // run: first place inside a block; end: of the sequence
    f32x4 bias;
    __device__ __forceinline__ Place(const RecurrenceArgs &a, uint32_t slab, uint32_t sequence)
        : ch(slab * kSlab + threadIdx.x % 16u * 4u, a.channels), b(sequence), run(threadIdx.x / 16u * L), length(a.length), end(a.length)
    {
        if (a.lengths) end = uint32_t(min(max(a.lengths[b], 0), int32_t(a.length)));
        bias = 0.f;
        if (a.bias) bias = ch.load(a.bias + ch.first);
    }
    template <typename S> __device__ __forceinline__ S *row(const StepsArgs &s, uint32_t t) const
    {
        return static_cast<S *>(const_cast<void *>(s.data)) + (int64_t(b) * s.batch + int64_t(t) * s.row + ch.first);
    }
    // the thread's places from t on; zeros behind the sequence's end
    __device__ __forceinline__ void load(raw4<T> (&to)[L], const StepsArgs &s, uint32_t t) const
    {
#pragma unroll
        for (int i = 0; i < L; ++i) to[i] = t + i < end && ch.live ? ch.load(row<const T>(s, t + i)) : raw4<T>{};
    }
    // m and 1 - a of place t
    template <bool RESETS> __device__ __forceinline__ void gates(const RecurrenceArgs &a, raw4<T> forget, uint32_t t, f32x4 &m, f32x4 &rest, f32x4 &on) const
    {
        const f32x4 f = widen4<T>(forget) + bias;
        const bool inside = t < end;
        const bool reset = RESETS && inside && a.resets[int64_t(b) * a.resets_stride + t] != 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const Gate g = state_gate_of(f[k]);
            on[k] = g.on;
            m[k] = !inside ? 1.f : reset ? 0.f : g.on;
            rest[k] = inside ? g.off : 0.f;
        }
    }
    __device__ __forceinline__ uint64_t state(uint32_t channels, uint64_t i) const { return i * channels + ch.first; }
};

template <typename T, int WAVES, int L, bool RESETS> __global__ __launch_bounds__(WAVES * 64) void k_recurrence_forward(RecurrenceArgs a)
{
    using P = Place<T, WAVES, L>;
    __shared__ Change room[2][WAVES][16];
    const P p(a, blockIdx.x % a.slabs, a.first_sequence + blockIdx.x / a.slabs);
    f32x4 carry = 0.f;
    if (a.first && p.ch.live) carry = p.ch.load(a.first + p.state(a.channels, p.b));
    uint32_t turn = 0;
    for (uint32_t block = 0; block < a.length; block += P::kSteps) {
        const uint32_t t0 = block + p.run;
        raw4<T> x[L], forget[L], out[L];
        p.load(x, a.x, t0);
        p.load(forget, a.forget, t0);
        if (a.out.data) p.load(out, a.out, t0);
        Change step[L], all = {1.f, 0.f};
#pragma unroll
        for (int i = 0; i < L; ++i) {
            f32x4 rest, on;
            p.template gates<RESETS>(a, forget[i], t0 + i, step[i].m, rest, on);
            step[i].v = rest * widen4<T>(x[i]);
            all.v = applied<RESETS>(step[i], all.v);
            all.m *= step[i].m;
        }
        f32x4 h = begin_of<WAVES, RESETS, false>(all, carry, room[turn]);
        turn ^= 1u;
        if (!p.ch.live) continue;
        if (a.states && t0 % ADACOMP_RECURRENCE_KEEP == 0u && t0 < a.length) p.ch.store(a.states + p.state(a.channels, uint64_t(p.b) * a.kept + t0 / ADACOMP_RECURRENCE_KEEP), h);
#pragma unroll
        for (int i = 0; i < L; ++i) {
            if (t0 + i >= a.length) break;
            h = applied<RESETS>(step[i], h);
            f32x4 y = h;
            if (a.out.data) {
                const f32x4 o = widen4<T>(out[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] *= gate_of<T>(o[k]).on;
            }
            if (t0 + i >= p.end) y = 0.f;
            p.ch.store(p.template row<T>(a.y, t0 + i), y);
        }
    }
    if (a.last && threadIdx.x < 16u && p.ch.live) p.ch.store(a.last + p.state(a.channels, p.b), carry);
}

template <typename T, int WAVES, int L, bool RESETS> __global__ __launch_bounds__(WAVES * 64) void k_recurrence_backward(RecurrenceArgs a)
{
    using P = Place<T, WAVES, L>;
    static_assert(P::kSteps % ADACOMP_RECURRENCE_KEEP == 0, "a block begins with a state that was kept");
    __shared__ Change room[2][2][WAVES][16];
    __shared__ f32x4 sums[WAVES * 4][16];
    const P p(a, blockIdx.x % a.slabs, a.first_sequence + blockIdx.x / a.slabs);
    f32x4 carry = 0.f, dbias = 0.f;
    if (a.first && p.ch.live) carry = p.ch.load(a.first + p.state(a.channels, p.b));
    uint32_t turn = 0;
    for (uint32_t blocks = a.length / P::kSteps + (a.length % P::kSteps != 0u); blocks-- > 0u;) {
        const uint32_t block = blocks * P::kSteps, t0 = block + p.run;
        raw4<T> x[L], forget[L], out[L], dy[L];
        p.load(x, a.x, t0);
        p.load(forget, a.forget, t0);
        p.load(dy, a.y, t0);
        if (a.out.data) p.load(out, a.out, t0);
        f32x4 state = 0.f;
        if (p.ch.live) state = p.ch.load(a.states + p.state(a.channels, uint64_t(p.b) * a.kept + block / ADACOMP_RECURRENCE_KEEP));
        f32x4 m[L], rest[L], on[L];
        Change all = {1.f, 0.f}, back = {1.f, 0.f};
#pragma unroll
        for (int i = 0; i < L; ++i) {
            p.template gates<RESETS>(a, forget[i], t0 + i, m[i], rest[i], on[i]);
            all.v = applied<RESETS>({m[i], rest[i] * widen4<T>(x[i])}, all.v);
            all.m *= m[i];
        }
        f32x4 d[L];
#pragma unroll
        for (int i = L - 1; i >= 0; --i) {
            d[i] = widen4<T>(dy[i]);
            if (a.out.data) {
                const f32x4 o = widen4<T>(out[i]);
#pragma unroll
                for (int k = 0; k < 4; ++k) d[i][k] *= gate_of<T>(o[k]).on;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) back.v[k] = through<RESETS>(m[i][k], d[i][k] + back.v[k]);
        }
        back.m = all.m;
        const f32x4 h0 = begin_of<WAVES, RESETS, false>(all, state, room[turn][0]);
        f32x4 c = begin_of<WAVES, RESETS, true>(back, carry, room[turn][1]);
        turn ^= 1u;
        f32x4 h[L];   // before each place
        h[0] = h0;
#pragma unroll
        for (int i = 1; i < L; ++i) h[i] = applied<RESETS>({m[i - 1], rest[i - 1] * widen4<T>(x[i - 1])}, h[i - 1]);
        if (p.ch.live) {
#pragma unroll
            for (int i = L - 1; i >= 0; --i) {
                if (t0 + i >= a.length) continue;
                const f32x4 g = d[i] + c, xi = widen4<T>(x[i]);
                f32x4 came, df, dout = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    came[k] = RESETS && m[i][k] == 0.f ? 0.f : h[i][k];
                    c[k] = through<RESETS>(m[i][k], g[k]);
                    df[k] = g[k] * (on[i][k] * rest[i][k]) * (came[k] - xi[k]);
                }
                const bool inside = t0 + i < p.end;
                if (a.out.data) {
                    const f32x4 o = widen4<T>(out[i]), up = widen4<T>(dy[i]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const Gate gate = gate_of<T>(o[k]);
                        dout[k] = up[k] * fmaf(m[i][k], came[k], rest[i][k] * xi[k]) * (gate.on * gate.off);
                    }
                    p.ch.store(p.template row<T>(a.dout, t0 + i), inside ? dout : f32x4(0.f));
                }
                if (!inside) df = 0.f;
                dbias += df;
                p.ch.store(p.template row<T>(a.dx, t0 + i), inside ? g * rest[i] : f32x4(0.f));
                p.ch.store(p.template row<T>(a.dforget, t0 + i), df);
            }
        }
    }
    if (a.last && threadIdx.x < 16u && p.ch.live) p.ch.store(a.last + p.state(a.channels, p.b), carry);
    if (!a.dbias_parts) return;
    sums[threadIdx.x / 16u][threadIdx.x % 16u] = dbias;
    __syncthreads();
    if (threadIdx.x >= 16u || !p.ch.live) return;
    f32x4 s = 0.f;
    for (uint32_t g = 0; g < WAVES * 4u; ++g) s += sums[g][threadIdx.x];
    p.ch.store(a.dbias_parts + p.state(a.channels, p.b), s);
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

constexpr int kWaves = 4, kRun = 4;

// Calls f with the arguments and the grid of every launch: a grid is counted in threads, in 32 bits.
template <typename F> static int for_sequences(const RecurrenceArgs &args, F &&f)
{
    RecurrenceArgs a = args;
    const uint32_t step = (1u << 23) / a.slabs;
    for (uint64_t first = 0; first < args.batch; first += step) {
        a.first_sequence = uint32_t(first);
        if (int rc = f(a, dim3(uint32_t(std::min<uint64_t>(step, args.batch - first)) * a.slabs))) return rc;
    }
    return ADACOMP_OK;
}

int launch_recurrence_forward(const RecurrenceArgs &args, uint32_t dtype, void *stream)
{
    const dim3 wg(kWaves * 64);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return for_sequences(args, [&](const RecurrenceArgs &a, dim3 grid) {
        return with_type(dtype, [&](auto of) {
            using T = decltype(of);
            if (a.resets) hipLaunchKernelGGL((k_recurrence_forward<T, kWaves, kRun, true>), grid, wg, 0, s, a);
            else hipLaunchKernelGGL((k_recurrence_forward<T, kWaves, kRun, false>), grid, wg, 0, s, a);
        });
    });
}

int launch_recurrence_backward(const RecurrenceArgs &args, uint32_t dtype, void *stream)
{
    const dim3 wg(kWaves * 64);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return for_sequences(args, [&](const RecurrenceArgs &a, dim3 grid) {
        return with_type(dtype, [&](auto of) {
            using T = decltype(of);
            if (a.resets) hipLaunchKernelGGL((k_recurrence_backward<T, kWaves, kRun, true>), grid, wg, 0, s, a);
            else hipLaunchKernelGGL((k_recurrence_backward<T, kWaves, kRun, false>), grid, wg, 0, s, a);
        });
    });
}

int launch_bias_sum(const BiasSumArgs &a, void *stream)
{
    hipLaunchKernelGGL(k_bias_sum, dim3((a.channels + 31u) / 32u), dim3(1024), 0, static_cast<hipStream_t>(stream), a);
    return check_launch();
}

}  // namespace adacomp
