// sequence_distill.hip -- kernels of the distillation loss and its gradient (adacomp_sequence.h).
//
// A row of logits belongs to a team of threads, which holds it in registers where it fits.  Every thread takes the maximum of its own
// logits off them and adds up exponentials, and the threads' sums are brought to the row's maximum when they are joined.  The
// teacher's top tokens are looked up beside that, in LDS.  Of the gradient first q is written, as if there were no teacher and no target, and
// then, behind a barrier, the few places that they speak about once more.
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

// What a team has in LDS: its row's top tokens, and behind them the target.
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

// Exponentials of one row at a temperature: of z less the row's maximum, or of z / temperature - lse.
template <typename T> struct Exponent {
    float off, c;
    bool minus_after;   // off is in units of z / temperature
    __device__ __forceinline__ float of(float z) const
    {
        if (minus_after) return exp_of<T>(z * c - off);
        return exp_of<T>((z - off) * c);
    }
};

__device__ __forceinline__ float finite_or_zero(float m) { return m == -kInf ? 0.f : m; }

// HELD: the row fits V groups of 8 to each thread; otherwise the team goes over it in parts, twice where it needs the maximum.
template <typename T, int TPR, int V, bool HELD, int PASS> __global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_distill(DistillArgs a)
{
    constexpr uint32_t TEAMS = TPR > 256 ? 1 : 256 / TPR, PART = TPR * V * 8;
    extern __shared__ float entries_room[];
    __shared__ float room[6][16];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>(), parts = HELD ? 1u : (a.vocab + PART - 1u) / PART;
    const Entries e(entries_room, team, a.top + 1u);
    const bool two = a.top != 0u && a.targets && a.per_temperature != 1.f;   // exponentials at both temperatures
    const float c = a.top != 0u ? a.per_temperature : 1.f;
    for (uint64_t first = uint64_t(blockIdx.x) * TEAMS; first < a.rows; first += uint64_t(gridDim.x) * TEAMS) {
        const uint64_t row = first + team;
        const bool live = row < a.rows;
        const T *z = static_cast<const T *>(a.logits) + row * a.logits_stride;
        auto groups_of = [&](uint32_t part) { return RowGroups<T, TPR, V>{t, a.vocab, part * PART}; };
        raw8<T> raw[V] = {};
        if (live) groups_of(0).load(raw, z);
        __syncthreads();   // the row before is done with the entries
        float top_max = -kInf;
        if (live)
            for (uint32_t k = t; k <= a.top; k += TPR) {
                uint32_t token = kNoToken;
                float tk = -kInf, zk = -kInf;
                if (k < a.top) {
                    token = token_of(a.teacher_tokens, row * a.tokens_stride + k, a.tokens64, a.vocab);
                    if (token != kNoToken) tk = value_of(a.teacher_logits, row * a.teacher_stride + k, a.teacher_dtype) * a.per_temperature;
                    if (tk > top_max || tk != tk) top_max = tk;   // a NaN stays
                } else if (a.targets) token = token_of(a.targets, row, a.targets64, a.vocab);
                if (token != kNoToken) zk = float(z[token]);
                e.token[k] = token;
                e.t[k] = tk;
                e.z[k] = zk;
            }
        // values of round v, -infinity behind the row's end
        auto values = [&](const RowGroups<T, TPR, V> &groups, int v) {
            f32x8 x = groups.values(raw[v], v);
            if (!groups.whole(v)) {
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = groups.col(v) + k < a.vocab ? x[k] : -kInf;
            }
            return x;
        };
        float most = -kInf, sum = 0.f, sum1 = 0.f;
        if constexpr (PASS != GRAD) {
            for (uint32_t part = 0; part < parts; ++part) {
                const RowGroups<T, TPR, V> groups = groups_of(part);
                if (part != 0u && live) groups.load(raw, z);
                float here = -kInf;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const f32x8 x = values(groups, v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) here = fmaxf(here, x[k]);
                }
                if (here > most) {
                    sum *= most == -kInf ? 1.f : exp_of<T>((most - here) * c);
                    if (two) sum1 *= most == -kInf ? 1.f : exp_of<T>(most - here);
                    most = here;
                }
                const Exponent<T> ex = {finite_or_zero(most), c, false}, ex1 = {ex.off, 1.f, false};
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const f32x8 x = values(groups, v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) sum += ex.of(x[k]);
                    if (two)
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum1 += ex1.of(x[k]);
                }
            }
            leave<Max, TPR>(most, room[0]);
        }
        leave<Max, TPR>(top_max, room[1]);
        __syncthreads();
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
            for (uint32_t k = t; k < a.top; k += TPR) {
                const float tk = e.t[k], p = exp_of<float>(tk - toff);
                s0 += p;
                if (PASS != GRAD && !(p == 0.f)) s1 += p * ((tk - toff) - (e.z[k] - zoff) * c);
                e.t[k] = p;
            }
        leave<Add, TPR>(s0, room[4]);
        if (PASS != GRAD) leave<Add, TPR>(s1, room[5]);
        __syncthreads();
        s0 = over_team<Add, TPR>(s0, room[4], team);
        const bool taught = !(s0 == 0.f), told = live && e.token[a.top] != kNoToken;
        float lse = 0.f, lse1 = 0.f, inv = 0.f, inv1 = 0.f;
        if constexpr (PASS != GRAD) {
            s1 = over_team<Add, TPR>(s1, room[5], team);
            sum = over_team<Add, TPR>(sum, room[2], team);
            sum1 = two ? over_team<Add, TPR>(sum1, room[3], team) : sum;
            inv = sum == 0.f || zmax * c == -kInf ? 0.f : 1.f / sum;
            inv1 = sum1 == 0.f ? 0.f : 1.f / sum1;
            const float log_sum = logf(sum), log_sum1 = two ? logf(sum1) : log_sum;
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
        Exponent<T> ex, ex1;
        if constexpr (PASS == GRAD) {   // a term that the row does not have: zeros
            ex = {two ? taught ? finite_or_zero(lse) : kInf : finite_or_zero(taught ? lse : lse1), c, true};
            ex1 = {told ? finite_or_zero(lse1) : kInf, 1.f, true};
            inv = inv1 = 1.f;
        } else {
            const float off = zmax * c == kInf ? __builtin_nanf("") : finite_or_zero(zmax);
            ex = {off, c, false};
            ex1 = {off, 1.f, false};
        }
        const float by = (two ? soft : soft + hard) * inv, by1 = hard * inv1;
        auto gradient = [&](float x) {
            float q = by * ex.of(x);
            if (two) q = fmaf(by1, ex1.of(x), q);
            return q;
        };
        T *dz = static_cast<T *>(a.dlogits) + row * a.dlogits_stride;
        if (live)
            for (uint32_t part = 0; part < parts; ++part) {
                const RowGroups<T, TPR, V> groups = groups_of(part);
                if (!HELD && (PASS != GRAD || part != 0u)) groups.load(raw, z);
                groups.store(dz, [&](int v) {
                    f32x8 x = groups.values(raw[v], v);
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = none ? 0.f : gradient(x[k]);
                    return x;
                });
            }
        __syncthreads();
        if (live && !none)
            for (uint32_t k = t; k <= a.top; k += TPR) {
                const uint32_t token = e.token[k];
                if (token == kNoToken) continue;
                float p = 0.f;
                if (taught)
                    for (uint32_t j = 0; j < a.top; ++j)
                        if (e.token[j] == token) p += e.t[j];
                float x = gradient(e.z[k]);
                if (taught) x -= soft * (p / s0);
                if (token == e.token[a.top]) x -= hard;
                dz[token] = T(x);
            }
    }
}

// ---- launches -----------------------------------------------------------------------------------------------------

// The entries of all teams are within 64 KB of LDS.
template <typename F> static void with_distill(uint32_t vocab, uint32_t top, F &&f)
{
    if (vocab <= 256u && top < 128u) f(std::integral_constant<int, 8>(), std::integral_constant<int, 4>(), std::true_type());
    else if (vocab <= 1024u) f(std::integral_constant<int, 32>(), std::integral_constant<int, 4>(), std::true_type());
    else if (vocab <= 4096u) f(std::integral_constant<int, 128>(), std::integral_constant<int, 4>(), std::true_type());
    else if (vocab <= 8192u) f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>(), std::true_type());
    else if (vocab <= 32768u) f(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>(), std::true_type());
    else f(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>(), std::false_type());
}

int launch_distill(const DistillArgs &a, uint32_t dtype, DistillPass pass, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto of) {
        using T = decltype(of);
        auto go = [&](auto which) {
            constexpr int PASS = decltype(which)::value;
            with_distill(a.vocab, a.top, [&](auto threads, auto groups, auto held) {
                constexpr uint32_t TPR = decltype(threads)::value, TEAMS = TPR > 256u ? 1u : 256u / TPR;
                const uint64_t blocks = (a.rows + TEAMS - 1u) / TEAMS;
                hipLaunchKernelGGL((k_distill<T, int(TPR), decltype(groups)::value, decltype(held)::value, PASS>), dim3(uint32_t(std::min<uint64_t>(blocks, 1u << 20))),
                                   dim3(std::max(TPR, 256u)), TEAMS * (a.top + 1u) * 12u, s, a);
            });
        };
        if (pass == LOSS) go(std::integral_constant<int, LOSS>());
        else if (pass == LOSS_GRAD) go(std::integral_constant<int, LOSS_GRAD>());
        else go(std::integral_constant<int, GRAD>());
    });
}

}  // namespace adacomp
