// sequence_distill.hip -- kernels of the distillation loss and its gradient (adacomp_sequence.h).
//
// A row of logits belongs to a team of threads, which goes over it in parts, or holds it in registers if it is short.  Every thread takes the maximum of its own
// logits off them and adds up exponentials, and the threads' sums are brought to the row's maximum when they are joined.  The
// teacher's top tokens are looked up beside that, in LDS.  Of the gradient first q is written, as if there were no teacher and no target, and
// then, behind a barrier, the few places that they speak about once more.
//
// Losses read the logits once: 4096 x 65536 bf16 100 us (5.4 TB/s).  The gradient reads and writes them once: the same 229 us (4.7 TB/s), 4099 x 50001, whose rows begin at
// odd addresses, 210 us (3.9 TB/s; 193 without the 101 places a row that are written again).  Loss and gradient at once read them twice, the second time from the
// memory-side cache for the most part: 4096 x 65536 291 us, where the two calls take 335; 5003 x 5999 f16 with two temperatures 37 us, bound by 33 vector instructions and 4
// exponentials a value.  Results of 16 bits go past the caches although some are written again: through them 4096 x 65536 takes 259 us.
// Cross entropy alone: 4096 x 65536 bf16 losses 100, both 271, the gradient 220 us; 32768 x 65 7.5, 12.3 and 9.9.  A row is never shared out over workgroups: 16 x 131072
// bf16 with 64 top tokens takes 11, 25 and 19 us.
#include "layers_device.h"
#include "sequence_plan.h"

namespace adacomp {

constexpr uint32_t kNoToken = 0xFFFFFFFFu;

__device__ __forceinline__ uint32_t token_of(const void *tokens, uint64_t i, uint32_t wide, uint32_t vocab)
{
    const int64_t t = wide ? static_cast<const int64_t *>(tokens)[i] : int64_t(static_cast<const int32_t *>(tokens)[i]);
    return uint64_t(t) < vocab ? uint32_t(t) : kNoToken;
}

__device__ __forceinline__ float value_of(const void *p, uint64_t i, uint32_t dtype)
{
    if (dtype == ADACOMP_DTYPE_F32) return static_cast<const float *>(p)[i];
    return dtype == ADACOMP_DTYPE_BF16 ? float(static_cast<const bf16 *>(p)[i]) : float(static_cast<const f16 *>(p)[i]);
}

// What a team has in LDS: its row's top tokens, and behind them the target and entries without a token, in fours.
__host__ __device__ constexpr uint32_t entry_pitch(uint32_t top) { return (top + 4u) & ~3u; }
struct Entries {
    uint32_t *token;
    float *t, *z;   // t / temperature, later p;  the student's logit
    __device__ __forceinline__ Entries(float *room, uint32_t team, uint32_t count)
        : token(reinterpret_cast<uint32_t *>(room) + team * 3u * count), t(room + (team * 3u + 1u) * count), z(room + (team * 3u + 2u) * count) {}
};

// Over the threads of a row, of which each wave of a larger team leaves its part in `room`.
template <typename OP, int TPR> __device__ __forceinline__ float over_team(float x, float *room, uint32_t team)
{
    if constexpr (TPR <= 64) return over_lanes<OP, TPR>(x);
    else {
        constexpr uint32_t WAVES = TPR / 64;
        x = room[team * WAVES];
#pragma unroll
        for (uint32_t w = 1; w < WAVES; ++w) x = OP::of(x, room[team * WAVES + w]);
        return x;
    }
}
template <typename OP, int TPR> __device__ __forceinline__ void leave(float x, float *room)
{
    if constexpr (TPR > 64) {
        x = over_lanes<OP, 64>(x);
        if (threadIdx.x % 64u == 0u) room[threadIdx.x / 64u] = x;
    }
}

// Exponentials of one row at a temperature: of (z - its maximum) / temperature, or of z / temperature - lse.  In 16 bits the factor and the change
// of units are one product; nothing but a difference is ever multiplied, so that logits at the ends of the type stay finite.
template <typename T, bool FROM_LSE> struct Exponent {
    float off, c;
    __device__ __forceinline__ Exponent(float o, float per) : off(o), c(!FROM_LSE && sizeof(T) == 2 ? per * kLog2e : per) {}
    __device__ __forceinline__ float of(float z) const
    {
        const float x = FROM_LSE ? fmaf(z, c, -off) : (z - off) * c;
        if constexpr (sizeof(T) == 4) return exp_of<T>(x);
        return __builtin_amdgcn_exp2f(FROM_LSE ? x * kLog2e : x);
    }
};

__device__ __forceinline__ float finite_or_zero(float m) { return m == -kInf ? 0.f : m; }

// Everything that the team's threads have stored, in LDS and in memory, is there for the others.  A wave's own accesses need no barrier, only their end.
template <int TPR> __device__ __forceinline__ void sync_team()
{
    if constexpr (TPR > 64) __syncthreads();
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}
// The same for LDS alone.
template <int TPR> __device__ __forceinline__ void sync_lds()
{
    if constexpr (TPR > 64) __syncthreads();
    else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// HELD: the row fits V groups of 8 to each thread; otherwise the team goes over it in parts, twice where it needs the maximum.
template <typename T, int TPR, int V, bool HELD, int PASS> __global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_distill(DistillArgs a)
{
    constexpr uint32_t TEAMS = TPR > 256 ? 1 : 256 / TPR, PART = TPR * V * 8;
    using Groups = RowGroups<T, TPR, V, kFlow<T>, DistillForm{TPR, V, HELD}.short_rows()>;
    extern __shared__ __attribute__((aligned(16))) float entries_room[];
    __shared__ float room[6][16];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>(), whole_parts = HELD ? 0u : a.vocab / PART;
    const uint32_t pitch = entry_pitch(a.top);
    const Entries e(entries_room, team, pitch);
    const bool two = a.top != 0u && a.targets && a.per_temperature != 1.f;   // exponentials at both temperatures
    const float c = a.top != 0u ? a.per_temperature : 1.f;
    for (uint64_t first = uint64_t(blockIdx.x) * TEAMS; first < a.rows; first += uint64_t(gridDim.x) * TEAMS) {
        const uint64_t row = first + team;
        const bool live = row < a.rows;
        const T *z = static_cast<const T *>(a.logits) + row * a.logits_stride;
        const Groups last = {t, a.vocab, whole_parts * PART};   // the part that the row ends in
        raw8<T> raw[V] = {};
        if (HELD && live) last.load(raw, z);
        // f(values) of every part: of whole ones, each with the next one on its way, and of the last one, where `behind` stands behind the row's end
        auto parts = [&](float behind, auto &&f) __attribute__((always_inline)) {
            if constexpr (!HELD) {
                if (!live) return;
                raw8<T> next[V];
                auto fetch = [&](uint32_t part) __attribute__((always_inline)) {
#pragma unroll
                    for (int v = 0; v < V; ++v) next[v] = load8(at(z, part * PART + (t + uint32_t(v) * TPR) * 8u));
                };
                if (whole_parts) fetch(0);
                for (uint32_t part = 0; part < whole_parts; ++part) {
                    f32x8 x[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) x[v] = widen<T>(next[v]);
                    fetch(min(part + 1u, whole_parts - 1u));
                    f(x, part * PART, std::true_type());
                }
                if (whole_parts * PART == a.vocab) return;
                last.load(raw, z);
            }
            f32x8 x[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[v] = last.values(raw[v], v);
                if (!last.whole(v)) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[v][k] = last.col(v) + k < a.vocab ? x[v][k] : behind;
                }
            }
            f(x, whole_parts * PART, std::false_type());
        };
        sync_lds<TPR>();   // the row before is done with the entries
        float top_max = -kInf;
        if (live)
            for (uint32_t k = t; k < pitch; k += TPR) {
                uint32_t token = kNoToken;
                float tk = -kInf, zk = -kInf;
                if (k < a.top) {
                    token = token_of(a.teacher_tokens, row * a.tokens_stride + k, a.tokens64, a.vocab);
                    if (token != kNoToken) tk = value_of(a.teacher_logits, row * a.teacher_stride + k, a.teacher_dtype) * a.per_temperature;
                    if (tk > top_max || tk != tk) top_max = tk;   // a NaN stays
                } else if (k == a.top && a.targets) token = token_of(a.targets, row, a.targets64, a.vocab);
                if (token != kNoToken) zk = float(z[token]);
                e.token[k] = token;
                e.t[k] = tk;
                e.z[k] = zk;
            }
        float most = -kInf, sum = 0.f, sum1 = 0.f;
        if constexpr (PASS != GRAD) {
            parts(-kInf, [&](const f32x8 (&x)[V], uint32_t, auto) __attribute__((always_inline)) {
                float here = -kInf;
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int k = 0; k < 8; ++k) here = fmaxf(here, x[v][k]);
                if (here > most) {
                    sum *= most == -kInf ? 1.f : exp_of<T>((most - here) * c);
                    if (two) sum1 *= most == -kInf ? 1.f : exp_of<T>(most - here);
                    most = here;
                }
                const Exponent<T, false> ex(finite_or_zero(most), c), ex1(ex.off, 1.f);
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum += ex.of(x[v][k]);
                if (two)
#pragma unroll
                    for (int v = 0; v < V; ++v)
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum1 += ex1.of(x[v][k]);
            });
            leave<Max, TPR>(most, room[0]);
        }
        leave<Max, TPR>(top_max, room[1]);
        sync_lds<TPR>();
        // fmaxf drops a NaN among the threads' maxima, but not in the sums, which then are NaN
        const float tmax = over_team<Max, TPR>(top_max, room[1], team), toff = finite_or_zero(tmax);
        float zmax = 0.f;
        if constexpr (PASS != GRAD) {
            zmax = over_team<Max, TPR>(most, room[0], team);
            sum *= most == -kInf ? 1.f : exp_of<T>((most - zmax) * c);
            if (two) sum1 *= most == -kInf ? 1.f : exp_of<T>(most - zmax);
            leave<Add, TPR>(sum, room[2]);
            if (two) leave<Add, TPR>(sum1, room[3]);
        }
        // of log p - log q what depends on the token, taken from the maxima: neither the logits nor lse may be large in it
        const float zoff = finite_or_zero(zmax);
        float s0 = 0.f, s1 = 0.f;
        if (live)
            for (uint32_t k = t; k < pitch; k += TPR) {
                const float tk = e.t[k], p = exp_of<float>(tk - toff);   // 0 of -infinity
                s0 += p;
                if (PASS != GRAD && !(p == 0.f)) s1 += p * ((tk - toff) - (e.z[k] - zoff) * c);
                e.t[k] = p;
            }
        leave<Add, TPR>(s0, room[4]);
        if (PASS != GRAD) leave<Add, TPR>(s1, room[5]);
        sync_lds<TPR>();
        s0 = over_team<Add, TPR>(s0, room[4], team);
        const bool taught = !(s0 == 0.f), told = live && e.token[a.top] != kNoToken;
        float lse = 0.f, lse1 = 0.f, inv = 0.f, inv1 = 0.f;
        if constexpr (PASS != GRAD) {
            s1 = over_team<Add, TPR>(s1, room[5], team);
            sum = over_team<Add, TPR>(sum, room[2], team);
            sum1 = two ? over_team<Add, TPR>(sum1, room[3], team) : sum;
            inv = sum == 0.f || zmax * c == -kInf ? 0.f : 1.f / sum;
            inv1 = sum1 == 0.f ? 0.f : 1.f / sum1;
            const float log_sum = zmax * c == kInf ? __builtin_nanf("") : logf(sum), log_sum1 = two ? logf(sum1) : log_sum;
            lse = zmax * c + log_sum;
            lse1 = zmax + log_sum1;
            if (live && t == 0u) {
                float loss = 0.f;
                if (taught) loss += a.soft_loss * (lse == -kInf ? kInf : s1 / s0 - logf(s0) + log_sum);
                if (told) loss += a.hard * (lse1 == -kInf ? kInf : log_sum1 - (e.z[a.top] - zoff));
                a.loss[row] = loss;
                if (a.lse) { a.lse[2u * row] = taught ? lse : 0.f; a.lse[2u * row + 1u] = told ? lse1 : 0.f; }
            }
        } else if (live) {
            lse = a.lse[2u * row];
            lse1 = a.lse[2u * row + 1u];
        }
        if constexpr (PASS == LOSS) continue;
        const float g = !live ? 0.f : a.dloss ? a.scale * a.dloss[row] : a.scale;
        const float soft = taught && g != 0.f ? g * a.soft_grad : 0.f, hard = told && g != 0.f ? g * a.hard : 0.f;
        const bool none = g == 0.f || !(taught || told);
        float off, off1;
        if constexpr (PASS == GRAD) {   // a term that the row does not have: zeros
            off = two ? taught ? finite_or_zero(lse) : kInf : finite_or_zero(taught ? lse : lse1);
            off1 = told ? finite_or_zero(lse1) : kInf;
            inv = inv1 = 1.f;
        } else {
            off = (taught || !two) && zmax * c == kInf ? __builtin_nanf("") : zoff;
            off1 = zmax == kInf ? __builtin_nanf("") : zoff;
        }
        const Exponent<T, PASS == GRAD> ex(off, c), ex1(off1, 1.f);
        const float by = (two ? soft : soft + hard) * inv, by1 = hard * inv1;
        auto gradient = [&](float x) {
            float q = by * ex.of(x);
            if (two) q = fmaf(by1, ex1.of(x), q);
            return q;
        };
        T *dz = static_cast<T *>(a.dlogits) + row * a.dlogits_stride;
        if (live)
            parts(0.f, [&](const f32x8 (&x)[V], uint32_t first_col, auto full) __attribute__((always_inline)) {
                constexpr bool FULL = decltype(full)::value;
                f32x8 y[V];
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[v][k] = none ? 0.f : gradient(x[v][k]);
                if constexpr (FULL) {
#pragma unroll
                    for (int v = 0; v < V; ++v) Groups::store_whole(at(dz, first_col + (t + uint32_t(v) * TPR) * 8u), y[v]);
                } else {
                    last.store(dz, [&](int v) { return y[v]; });
                }
            });
        sync_team<TPR>();
        if (live && !none)
            for (uint32_t k = t; k <= a.top; k += TPR) {
                const uint32_t token = e.token[k];
                if (token == kNoToken) continue;
                float p = 0.f;
                if (taught)
#pragma unroll 2
                    for (uint32_t j = 0; j < pitch; j += 4u) {
                        const uint4 others = *reinterpret_cast<const uint4 *>(e.token + j);
                        const float4 ps = *reinterpret_cast<const float4 *>(e.t + j);
                        p += others.x == token ? ps.x : 0.f;
                        p += others.y == token ? ps.y : 0.f;
                        p += others.z == token ? ps.z : 0.f;
                        p += others.w == token ? ps.w : 0.f;
                    }
                float x = gradient(e.z[k]);
                if (taught) x -= soft * (p / s0);
                if (token == e.token[a.top]) x -= hard;
                dz[token] = T(x);
            }
    }
}

// ---- launches -----------------------------------------------------------------------------------------------------

template <typename F> static void with_distill(const DistillForm &form, F &&f)
{
    using One = std::integral_constant<int, 1>;
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (form.threads == 8u) f(std::integral_constant<int, 8>(), Four(), std::true_type());
    else if (form.threads == 32u && form.groups == 1u) f(std::integral_constant<int, 32>(), One(), std::true_type());
    else if (form.threads == 32u) f(std::integral_constant<int, 32>(), Four(), std::true_type());
    else if (form.threads == 64u) f(std::integral_constant<int, 64>(), Two(), std::false_type());
    else if (form.threads == 256u) f(std::integral_constant<int, 256>(), Two(), std::false_type());
    else f(std::integral_constant<int, 1024>(), Two(), std::false_type());
}

int launch_distill(const DistillArgs &a, uint32_t dtype, DistillPass pass, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto of) {
        using T = decltype(of);
        auto go = [&](auto which) {
            constexpr int PASS = decltype(which)::value;
            with_distill(distill_form(a.rows, a.vocab, a.top), [&](auto threads, auto groups, auto held) {
                constexpr uint32_t TPR = decltype(threads)::value, TEAMS = TPR > 256u ? 1u : 256u / TPR;
                const uint64_t blocks = (a.rows + TEAMS - 1u) / TEAMS;
                hipLaunchKernelGGL((k_distill<T, int(TPR), decltype(groups)::value, decltype(held)::value, PASS>), dim3(uint32_t(std::min<uint64_t>(blocks, 1u << 20))),
                                   dim3(std::max(TPR, 256u)), TEAMS * entry_pitch(a.top) * 12u, s, a);
            });
        };
        if (pass == LOSS) go(std::integral_constant<int, LOSS>());
        else if (pass == LOSS_GRAD) go(std::integral_constant<int, LOSS_GRAD>());
        else go(std::integral_constant<int, GRAD>());
    });
}

}  // namespace adacomp
