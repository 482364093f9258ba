// layers_norm.hip -- kernels of dropout and layer norm (adacomp_layers.h).
#include "layers_device.h"

namespace adacomp {

// ---- dropout ------------------------------------------------------------------------------------------------------
// y = [residual +] D(x).  One group of 8 columns to a thread and round; rows are cut into groups of their own, so that a
// group is one counter wherever it lies.

constexpr uint32_t kDropRounds = 4;

template <typename T> __global__ __launch_bounds__(256) void k_dropout(DropoutLaunch a)
{
    const Drop d = drop_of(a.drop);
    const uint32_t total = a.rows * a.groups;
#pragma unroll
    for (uint32_t u = 0; u < kDropRounds; ++u) {
        const uint32_t g = (blockIdx.x * kDropRounds + u) * 256u + threadIdx.x;
        if (g >= total) break;
        const uint32_t r = g / a.groups, c = g - r * a.groups;
        const uint64_t row = a.first_row + r;
        const uint32_t n = a.cols - c * 8u;
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride + c * 8ull, *res = static_cast<const T *>(a.residual) + row * a.residual_stride + c * 8ull;
        T *y = static_cast<T *>(a.y) + row * a.y_stride + c * 8ull;
        raw8<T> raw = {}, raw_res = {};
        if (n >= 8u) {
            raw = load8(x);
            if (a.residual) raw_res = load8(res);
        } else {
            raw = load_some(x, n);
            if (a.residual) raw_res = load_some(res, n);
        }
        f32x8 v = drop8(widen<T>(raw), d, c, uint32_t(row));
        if (a.residual) v += widen<T>(raw_res);
        if (n >= 8u) store8(y, v);
        else store_some(y, n, v);
    }
}

// ---- layer norm, forward ------------------------------------------------------------------------------------------
// A row stays in the registers of its threads: mean first, then the squared distances from it.

// Over the TPR threads of a row.  A row of several waves joins their sums in `room`, of which the next call takes another one.
template <int TPR> __device__ __forceinline__ float over_row(float x, float *room, uint32_t team)
{
    if constexpr (TPR <= 64) return over_lanes<Add, TPR>(x);
    else {
        constexpr uint32_t WAVES = TPR / 64;
        x = over_lanes<Add, 64>(x);
        if (threadIdx.x % 64u == 0u) room[threadIdx.x / 64u] = x;
        __syncthreads();
        x = room[team * WAVES];
#pragma unroll
        for (uint32_t w = 1; w < WAVES; ++w) x += room[team * WAVES + w];
        return x;
    }
}

template <typename T, int TPR, int V> __global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_norm_forward(NormForward a)
{
    constexpr uint32_t TEAMS = TPR > 256 ? 1 : 256 / TPR;
    __shared__ float room[2][16];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>();
    const Drop d = drop_of(a.drop);
    for (uint32_t first = blockIdx.x * TEAMS; first < a.rows; first += gridDim.x * TEAMS) {
        const bool live = first + team < a.rows;
        const uint32_t row = live ? first + team : a.rows - 1u;   // the last rows' workgroup has teams without one: they go along
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        const uint32_t cols = again_uniform(a.cols);
        const RowGroups<T, TPR, V> groups = {again(t), cols, 0};
        const RowGroups<float, TPR, V> params = {groups.t, cols, 0};
        const Drop dr = again(d);
        raw8<T> raw[V], raw_res[V];
        groups.load(raw, x);
        if (a.residual) groups.load(raw_res, static_cast<const T *>(a.residual) + row * a.residual_stride);
        raw8<float> some_gamma, some_beta;
        if (a.gamma) some_gamma = params.some(a.gamma);
        if (a.beta) some_beta = params.some(a.beta);
        raw8<float> gamma[V], beta[V];   // up to 8192 columns on their way together with the row, in wider rows behind its sums
        if constexpr (V == 1) {
            if (a.gamma) gamma[0] = params.round(a.gamma, 0, some_gamma);
            if (a.beta) beta[0] = params.round(a.beta, 0, some_beta);
        }
        f32x8 z[V];
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            z[v] = widen<T>(raw[v]);
            if (a.drop.on) z[v] = drop8(z[v], dr, groups.col(v) / 8u, row);
            if (a.residual) z[v] += widen<T>(raw_res[v]);
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += z[v][k];
        }
        const float mean = over_row<TPR>(sum, room[0], team) / float(a.cols);
        float squares = 0.f;
        f32x8 c[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            c[v] = z[v] - mean;
            if (!groups.whole(v)) {   // nothing behind the row's end counts
#pragma unroll
                for (int k = 0; k < 8; ++k) c[v][k] = groups.col(v) + k < cols ? c[v][k] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) squares = fmaf(c[v][k], c[v][k], squares);
        }
        const float rstd = 1.f / sqrtf(over_row<TPR>(squares, room[1], team) / float(a.cols) + a.eps);
        if (!live) continue;
        if (t == 0u) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        if (a.z) groups.store(static_cast<T *>(a.z) + row * a.z_stride, [&](int v) { return z[v]; });
        groups.store(static_cast<T *>(a.y) + row * a.y_stride, [&](int v) {
            f32x8 y = c[v] * rstd;
            if constexpr (V > 1) {
                if (a.gamma) gamma[v] = params.round(a.gamma, v, some_gamma);
                if (a.beta) beta[v] = params.round(a.beta, v, some_beta);
            }
            if (a.gamma) y *= gamma[v];
            if (a.beta) y += beta[v];
            return y;
        });
    }
}

// ---- layer norm, backward -----------------------------------------------------------------------------------------
// A workgroup of 1024 threads walks over rows, each held in registers as in the forward pass, with the next ones on their way, and
// keeps its columns' sums of dy h and of dy in registers until its last row; k_norm_reduce adds the workgroups' sums up.  Their
// traffic is 16 bytes a column and workgroup: large workgroups, one to a compute unit, keep it small beside the rows' 8 to 20.

constexpr uint32_t kBackThreads = 1024;

template <typename T, int TPR, int V> __global__ __launch_bounds__(kBackThreads) void k_norm_backward(NormBackward a)
{
    constexpr uint32_t TEAMS = kBackThreads / TPR, COLS = TPR * V * 8;
    __shared__ float room[2][2][16];
    __shared__ float sums[TEAMS > 1 ? TEAMS * COLS : 1];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>();
    const Drop d = drop_of(a.drop);
    const float per_col = 1.f / float(a.cols);
    f32x8 dgamma[V] = {}, dbeta[V] = {};
    raw8<float> gamma[V];
    if (a.gamma) RowGroups<float, TPR, V>{t, a.cols, 0}.load(gamma, a.gamma);
    raw8<T> raw_dy[V], raw_z[V], raw_add[V];
    float mean = 0.f, rstd = 0.f;
    auto fetch = [&](uint32_t row) {
        const RowGroups<T, TPR, V> groups = {again(t), again_uniform(a.cols), 0};
#pragma unroll
        for (int v = 0; v < V; ++v) raw_dy[v] = raw_z[v] = raw_add[v] = raw8<T>{};
        if (row < a.rows) {
            groups.load(raw_dy, static_cast<const T *>(a.dy) + row * a.dy_stride);
            groups.load(raw_z, static_cast<const T *>(a.z) + row * a.z_stride);
            if (a.dz_add) groups.load(raw_add, static_cast<const T *>(a.dz_add) + row * a.dz_add_stride);
            mean = a.mean[row];
            rstd = a.rstd[row];
        }
    };
    uint32_t turn = 0;
    fetch(blockIdx.x * TEAMS + team);
    for (uint32_t first = blockIdx.x * TEAMS; first < a.rows; first += gridDim.x * TEAMS) {
        const uint32_t row = first + team;
        const float scale = rstd;
        f32x8 g[V], h[V], dz[V];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            g[v] = widen<T>(raw_dy[v]);
            h[v] = (widen<T>(raw_z[v]) - mean) * scale;
            dz[v] = widen<T>(raw_add[v]);
            dbeta[v] += g[v];
#pragma unroll
            for (int k = 0; k < 8; ++k) dgamma[v][k] = fmaf(g[v][k], h[v][k], dgamma[v][k]);
            if (a.gamma) g[v] *= gamma[v];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                s1 += g[v][k];   // behind the row's end, and in teams without a row, g is 0
                s2 = fmaf(g[v][k], h[v][k], s2);
            }
        }
        fetch(row + gridDim.x * TEAMS);
        if constexpr (TPR <= 64) {
            s1 = over_lanes<Add, TPR>(s1);
            s2 = over_lanes<Add, TPR>(s2);
        } else {
            constexpr uint32_t WAVES = TPR / 64;
            s1 = over_lanes<Add, 64>(s1);
            s2 = over_lanes<Add, 64>(s2);
            if (threadIdx.x % 64u == 0u) { room[turn][0][threadIdx.x / 64u] = s1; room[turn][1][threadIdx.x / 64u] = s2; }
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < WAVES; ++w) { s1 += room[turn][0][team * WAVES + w]; s2 += room[turn][1][team * WAVES + w]; }
            turn ^= 1u;
        }
        if (row >= a.rows) continue;
        s1 *= per_col;
        s2 *= per_col;
        const RowGroups<T, TPR, V> groups = {again(t), again_uniform(a.cols), 0};
        const Drop dr = again(d);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int k = 0; k < 8; ++k) dz[v][k] = fmaf(scale, g[v][k] - fmaf(h[v][k], s2, s1), dz[v][k]);
        groups.store(static_cast<T *>(a.dz) + row * a.dz_stride, [&](int v) { return dz[v]; });
        if (a.dx) groups.store(static_cast<T *>(a.dx) + row * a.dx_stride, [&](int v) { return drop8(dz[v], dr, groups.col(v) / 8u, row); });
    }
    float *out = a.partial;
    if (!out) return;
    out += uint64_t(blockIdx.x) * 2u * a.pitch;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (TEAMS > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v)
                *reinterpret_cast<f32x8 *>(&sums[team * COLS + (t + v * TPR) * 8u]) = which ? dbeta[v] : dgamma[v];
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < a.pitch; c += kBackThreads) {
                float s = 0.f;
#pragma unroll 8
                for (uint32_t m = 0; m < TEAMS; ++m) s += sums[m * COLS + c];
                out[which * a.pitch + c] = s;
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t c = (t + v * TPR) * 8u;
                if (c < a.pitch) *reinterpret_cast<f32x8 *>(out + which * a.pitch + c) = which ? dbeta[v] : dgamma[v];
            }
        }
    }
}

// 32 columns to a workgroup, 32 slices of the parts; always in the same order.
__global__ __launch_bounds__(1024) void k_norm_reduce(NormReduce a)
{
    __shared__ float sums[32][33];
    const uint32_t lane = threadIdx.x % 32u, slice = threadIdx.x / 32u;
    const uint32_t c = blockIdx.x * 32u + lane, which = blockIdx.y;
    float s = 0.f;
    if (c < a.cols)
#pragma unroll 8
        for (uint32_t p = slice; p < a.parts; p += 32u) s += a.partial[(uint64_t(p) * 2u + which) * a.pitch + c];
    sums[slice][lane] = s;
    __syncthreads();
    if (slice != 0u || c >= a.cols) return;
    float *out = which ? a.dbeta : a.dgamma;
    if (!out) return;
    float all = 0.f;
    for (uint32_t k = 0; k < 32u; ++k) all += sums[k][lane];
    out[c] = a.accumulate ? out[c] + all : all;
}

// ---- launches -----------------------------------------------------------------------------------------------------

static int check_launch() { return hipGetLastError() == hipSuccess ? ADACOMP_OK : ADACOMP_EHIP; }

int launch_dropout(const DropoutLaunch &a, void *stream)
{
    const uint32_t total = a.rows * a.groups, per = 256u * kDropRounds;
    const dim3 grid((total + per - 1u) / per), wg(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.dtype == ADACOMP_DTYPE_F32) hipLaunchKernelGGL(k_dropout<float>, grid, wg, 0, s, a);
    else if (a.dtype == ADACOMP_DTYPE_BF16) hipLaunchKernelGGL(k_dropout<bf16>, grid, wg, 0, s, a);
    else hipLaunchKernelGGL(k_dropout<f16>, grid, wg, 0, s, a);
    return check_launch();
}

// 8 values to a thread as far as 1024 threads hold the row.
RowForm norm_form(uint32_t cols)
{
    uint32_t threads = 8;
    while (threads < 1024u && threads * 8u < cols) threads *= 2u;
    return {threads, cols <= 8192u ? 1u : cols <= 16384u ? 2u : 4u};
}

constexpr uint32_t kMostWorkgroups = 1u << 20;   // a launch has fewer than 2^32 threads; more rows are walked over

uint32_t norm_parts(uint64_t rows, uint32_t cols)
{
    const uint32_t teams = kBackThreads / norm_form(cols).threads;
    return uint32_t(std::min<uint64_t>((rows + teams - 1u) / teams, kComputeUnits));
}

template <template <typename, int, int> class K, typename A>
static int launch_rows(const RowForm &f, uint32_t dtype, uint32_t workgroups, uint32_t threads, const A &a, void *stream)
{
    const dim3 grid(workgroups), wg(threads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto go = [&](auto form) {
        constexpr int TPR = decltype(form)::threads, V = decltype(form)::groups;
        if (dtype == ADACOMP_DTYPE_F32) hipLaunchKernelGGL((K<float, TPR, V>::kernel), grid, wg, 0, s, a);
        else if (dtype == ADACOMP_DTYPE_BF16) hipLaunchKernelGGL((K<bf16, TPR, V>::kernel), grid, wg, 0, s, a);
        else hipLaunchKernelGGL((K<f16, TPR, V>::kernel), grid, wg, 0, s, a);
    };
    switch (f.threads * f.groups) {
    case 8: go(FormOf<8, 1>()); break;
    case 16: go(FormOf<16, 1>()); break;
    case 32: go(FormOf<32, 1>()); break;
    case 64: go(FormOf<64, 1>()); break;
    case 128: go(FormOf<128, 1>()); break;
    case 256: go(FormOf<256, 1>()); break;
    case 512: go(FormOf<512, 1>()); break;
    case 1024: go(FormOf<1024, 1>()); break;
    case 2048: go(FormOf<1024, 2>()); break;
    case 4096: go(FormOf<1024, 4>()); break;
    default: return ADACOMP_EINVAL;
    }
    return check_launch();
}

template <typename T, int TPR, int V> struct KForward { static constexpr auto kernel = k_norm_forward<T, TPR, V>; };
template <typename T, int TPR, int V> struct KBackward { static constexpr auto kernel = k_norm_backward<T, TPR, V>; };

int launch_norm_forward(const NormForward &a, uint32_t dtype, void *stream)
{
    const RowForm f = norm_form(a.cols);
    return launch_rows<KForward>(f, dtype, std::min((a.rows + f.teams() - 1u) / f.teams(), kMostWorkgroups), f.workgroup(), a, stream);
}

int launch_norm_backward(const NormBackward &a, uint32_t dtype, uint32_t parts, void *stream)
{
    return launch_rows<KBackward>(norm_form(a.cols), dtype, parts, kBackThreads, a, stream);
}

int launch_norm_reduce(const NormReduce &a, void *stream)
{
    hipLaunchKernelGGL(k_norm_reduce, dim3((a.cols + 31u) / 32u, 2), dim3(1024), 0, static_cast<hipStream_t>(stream), a);
    return check_launch();
}

}  // namespace adacomp
