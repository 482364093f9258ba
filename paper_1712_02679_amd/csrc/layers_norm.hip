// layers_norm.hip -- kernels of dropout and layer norm (adacomp_layers.h).
//
// All of them read each input once and write each result once (rows of more than 8192 columns are read twice in the backward pass, the
// second time from the caches), and are bound by memory in large calls, by one chain of load, reductions and store in small ones.
// 16384 x 4096 bf16: residual sum with dropout 64 us (6.3 TB/s), norm with both and its z 93 us (5.8 TB/s), backward with both 118 us (5.7 TB/s,
// of which k_norm_reduce 5); one row of 4096 3.1 us; 6007 x 577 f32 8.1 and 14.7 us.
// The backward pass that reads twice is further off: 8192 x 8200 bf16 166 us (2.4 TB/s), 8192 x 16384 238 us (3.4), 4096 x 32768 615 us (1.3); the last
// is the form for more than 16384 columns, which spills 94 to 98 vector registers to memory.
#include "layers_device.h"

namespace adacomp {

// ---- dropout ------------------------------------------------------------------------------------------------------
// y = [residual +] D(x).  One group of 8 columns to a thread (2 and 4 were slower: 71.5, 76.4 us to 70.0 at 16384 x 4096 bf16, and 3.6, 5.2 to 2.6 at
// 100 x 500 f32); rows are cut into groups of their own, so that a group is one counter wherever it lies.

template <typename T, bool ONCE> __global__ __launch_bounds__(256) void k_dropout(DropoutLaunch a)
{
    const Drop d = drop_of(a.drop);
    const uint32_t g = blockIdx.x * 256u + threadIdx.x;
    if (g >= a.rows * a.groups) return;
    const uint32_t r = g / a.groups, c = g - r * a.groups;
    const uint64_t row = a.first_row + r, col = c * 8ull;
    const uint32_t n = a.cols - c * 8u, back = a.cols < 8u || n >= 8u ? 0u : 8u - n;   // an incomplete group reads the row's last 8 values
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride + col - back, *res = static_cast<const T *>(a.residual) + row * a.residual_stride + col - back;
    raw8<T> raw, raw_res = {};
    if constexpr (ONCE) {
        raw = load8_once(x);
        if (a.residual) raw_res = load8_once(res);
    } else if (a.cols >= 8u) {
        raw = load8(x);
        if (a.residual) raw_res = load8(res);
    } else {
        raw = load_some(x, n);
        if (a.residual) raw_res = load_some(res, n);
    }
    f32x8 v = widen<T>(raw), w = widen<T>(raw_res);
    if (back) {
        v = shifted(v, 8u - a.cols % 8u);
        w = shifted(w, 8u - a.cols % 8u);
    }
    v = drop8(v, d, c, uint32_t(row));
    if (a.residual) v += w;
    T *y = static_cast<T *>(a.y) + row * a.y_stride + col;
    if (n >= 8u && sizeof(T) == 2) store8_past(y, v);
    else if (n >= 8u) store8(y, v);
    else store_some(y, n, v);
}

// ---- layer norm, forward ------------------------------------------------------------------------------------------
// A row stays in the registers of its threads: mean first, then the squared distances from it.  One row to a team of threads and no
// loop: workgroups that walk over rows with the next one on its way were slower (4096 columns 108 us to 98), and so was fetching gamma and
// beta ahead of the sums, which takes the registers of three waves in eight (bf16 59 / 61 us without residual).

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

template <typename T, int TPR, int V, int FLOW> __global__ __launch_bounds__(TPR > 256 ? TPR : 256) void k_norm_forward(NormForward a)
{
    constexpr uint32_t TEAMS = TPR > 256 ? 1 : 256 / TPR;
    __shared__ float room[2][16];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>(), row = blockIdx.x * TEAMS + team;
    const bool live = row < a.rows;   // the last workgroup may have teams without a row: they go along to the barriers
    const RowGroups<T, TPR, V, FLOW> groups = {t, a.cols, 0};
    raw8<T> raw[V] = {}, raw_res[V] = {};
    if (live) {
        groups.load(raw, static_cast<const T *>(a.x) + row * a.x_stride);
        if (a.residual) groups.load(raw_res, static_cast<const T *>(a.residual) + row * a.residual_stride);
    }
    const Drop d = drop_of(a.drop);
    f32x8 z[V];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        z[v] = groups.values(raw[v], v);
        if (a.drop.on) z[v] = drop8(z[v], d, groups.col(v) / 8u, uint32_t(a.first_row) + row);
        if (a.residual) z[v] += groups.values(raw_res[v], v);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += z[v][k];
    }
    const float mean = over_row<TPR>(sum, room[0], team) / float(a.cols);
    float squares = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        f32x8 c = z[v] - mean;
        if (!groups.whole(v)) {   // nothing behind the row's end counts
#pragma unroll
            for (int k = 0; k < 8; ++k) c[k] = groups.col(v) + k < a.cols ? c[k] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) squares = fmaf(c[k], c[k], squares);
    }
    const float rstd = 1.f / sqrtf(over_row<TPR>(squares, room[1], team) / float(a.cols) + a.eps);
    if (!live) return;
    if (t == 0u) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    if (a.z) groups.store(static_cast<T *>(a.z) + row * a.z_stride, [&](int v) { return z[v]; });
    const RowGroups<float, TPR, V> params = {t, a.cols, 0};
    groups.store(static_cast<T *>(a.y) + row * a.y_stride, [&](int v) {
        f32x8 y = (z[v] - mean) * rstd;
        if (a.gamma) y *= params.values(params.load_round(a.gamma, v), v);
        if (a.beta) y += params.values(params.load_round(a.beta, v), v);
        return y;
    });
}

// ---- layer norm, backward -----------------------------------------------------------------------------------------
// A workgroup of 1024 threads walks over rows, each held in registers as in the forward pass, with the next ones on their way, and
// keeps its columns' sums of dy h and of dy in registers until its last row; k_norm_reduce adds the workgroups' sums up.  Their
// traffic is 16 bytes a column and workgroup: large workgroups, one to a compute unit, keep it small beside the rows' 8 to 20.

constexpr uint32_t kBackThreads = 1024;

template <typename T, int TPR, int FLOW> __global__ __launch_bounds__(kBackThreads) void k_norm_backward(NormBackward a)
{
    constexpr uint32_t TEAMS = kBackThreads / TPR, COLS = TPR * 8;
    __shared__ float room[2][2][16];
    __shared__ alignas(32) float sums[TEAMS > 1 ? TEAMS * COLS : 8];
    const uint32_t t = threadIdx.x % TPR, team = team_of<TPR>();
    const Drop d = drop_of(a.drop);
    const float per_col = 1.f / float(a.cols);
    f32x8 dgamma = 0.f, dbeta = 0.f, gamma = 1.f;
    if (a.gamma) {
        const RowGroups<float, TPR, 1> params = {t, a.cols, 0};
        gamma = params.values(params.load_round(a.gamma, 0), 0);
    }
    raw8<T> raw_dy, raw_z, raw_add;
    float mean = 0.f, rstd = 0.f;
    auto fetch = [&](uint32_t row) {
        const RowGroups<T, TPR, 1, FLOW> groups = {again(t), again_uniform(a.cols), 0};
        raw_dy = raw_z = raw_add = raw8<T>{};
        if (row < a.rows) {
            raw_dy = groups.load_round(static_cast<const T *>(a.dy) + row * a.dy_stride, 0);
            raw_z = groups.load_round(static_cast<const T *>(a.z) + row * a.z_stride, 0);
            if (a.dz_add) raw_add = groups.load_round(static_cast<const T *>(a.dz_add) + row * a.dz_add_stride, 0);
            mean = a.mean[row];
            rstd = a.rstd[row];
        }
    };
    uint32_t turn = 0;
    fetch(blockIdx.x * TEAMS + team);
    for (uint32_t first = blockIdx.x * TEAMS; first < a.rows; first += gridDim.x * TEAMS) {
        const uint32_t row = first + team;
        const float scale = rstd;
        const RowGroups<T, TPR, 1, FLOW> groups = {again(t), again_uniform(a.cols), 0};
        f32x8 g = groups.values(raw_dy, 0), dz = groups.values(raw_add, 0);
        const f32x8 h = (groups.values(raw_z, 0) - mean) * scale;
        fetch(row + gridDim.x * TEAMS);
        float s1 = 0.f, s2 = 0.f;
        dbeta += g;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            dgamma[k] = fmaf(g[k], h[k], dgamma[k]);
            g[k] *= gamma[k];   // behind the row's end, and in teams without a row, g is 0
            s1 += g[k];
            s2 = fmaf(g[k], h[k], s2);
        }
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
#pragma unroll
        for (int k = 0; k < 8; ++k) dz[k] = fmaf(scale, g[k] - fmaf(h[k], s2, s1), dz[k]);
        groups.store(static_cast<T *>(a.dz) + row * a.dz_stride, [&](int) { return dz; });
        if (a.dx) groups.store(static_cast<T *>(a.dx) + row * a.dx_stride, [&](int) { return drop8(dz, again(d), groups.col(0) / 8u, row); });
    }
    if (!a.partial) return;
    float *out = a.partial + uint64_t(blockIdx.x) * 2u * a.pitch;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (TEAMS > 1) {
            __syncthreads();
            *reinterpret_cast<f32x8 *>(&sums[team * COLS + t * 8u]) = which ? dbeta : dgamma;
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < a.pitch; c += kBackThreads) {
                float s = 0.f;
#pragma unroll 8
                for (uint32_t m = 0; m < TEAMS; ++m) s += sums[m * COLS + c];
                out[which * a.pitch + c] = s;
            }
        } else if (t * 8u < a.pitch) {
            store8(out + which * a.pitch + t * 8u, which ? dbeta : dgamma);
        }
    }
}

// Rows of more than 8192 columns: the sums of V groups of columns leave no registers for the row, which is read a second time, from
// the caches, for dz.  With 4 groups the sums alone take 64 of a thread's 128 registers, and what does not fit beside them is spilled.
template <typename T, int V> __global__ __launch_bounds__(kBackThreads) void k_norm_backward_wide(NormBackward a)
{
    constexpr int TPR = kBackThreads;
    __shared__ float room[2][16];
    const uint32_t t = threadIdx.x;
    const Drop d = drop_of(a.drop);
    const float per_col = 1.f / float(a.cols);
    f32x8 dgamma[V] = {}, dbeta[V] = {};
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride, *z = static_cast<const T *>(a.z) + row * a.z_stride;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const RowGroups<T, TPR, V> groups = {again(t), again_uniform(a.cols), 0};
            const RowGroups<float, TPR, V> params = {groups.t, groups.cols, 0};
            f32x8 g = groups.values(groups.load_round(dy, v), v);
            const f32x8 h = (groups.values(groups.load_round(z, v), v) - mean) * rstd;
            dbeta[v] += g;
#pragma unroll
            for (int k = 0; k < 8; ++k) dgamma[v][k] = fmaf(g[k], h[k], dgamma[v][k]);
            if (a.gamma) g *= params.values(params.load_round(a.gamma, v), v);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                s1 += g[k];
                s2 = fmaf(g[k], h[k], s2);
            }
        }
        s1 = over_waves<Add, TPR / 64>(over_lanes<Add, 64>(s1), room[0]) * per_col;
        s2 = over_waves<Add, TPR / 64>(over_lanes<Add, 64>(s2), room[1]) * per_col;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const RowGroups<T, TPR, V> groups = {again(t), again_uniform(a.cols), 0};
            const RowGroups<float, TPR, V> params = {groups.t, groups.cols, 0};
            f32x8 g = groups.values(groups.load_round(dy, v), v), dz = 0.f;
            const f32x8 h = (groups.values(groups.load_round(z, v), v) - mean) * rstd;
            if (a.gamma) g *= params.values(params.load_round(a.gamma, v), v);
            if (a.dz_add) dz = groups.values(groups.load_round(static_cast<const T *>(a.dz_add) + row * a.dz_add_stride, v), v);
#pragma unroll
            for (int k = 0; k < 8; ++k) dz[k] = fmaf(rstd, g[k] - fmaf(h[k], s2, s1), dz[k]);
            groups.store_round(static_cast<T *>(a.dz) + row * a.dz_stride, v, dz);
            if (a.dx) groups.store_round(static_cast<T *>(a.dx) + row * a.dx_stride, v, drop8(dz, again(d), groups.col(v) / 8u, row));
        }
    }
    if (!a.partial) return;
    float *out = a.partial + uint64_t(blockIdx.x) * 2u * a.pitch;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const uint32_t c = (t + v * TPR) * 8u;
        if (c >= a.pitch) continue;
        store8(out + c, dgamma[v]);
        store8(out + a.pitch + c, dbeta[v]);
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

// Whether all of a tensor's rows begin with a line of memory.
static bool lines(const void *p, uint64_t stride, uint64_t size) { return !p || (reinterpret_cast<uintptr_t>(p) | stride * size) % 64u == 0u; }

int launch_dropout(const DropoutLaunch &a, void *stream)
{
    const dim3 grid((a.rows * a.groups + 255u) / 256u), wg(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint64_t size = a.dtype == ADACOMP_DTYPE_F32 ? 4u : 2u;
    const bool once = size == 2u && a.cols % 32u == 0u && lines(a.x, a.x_stride, size) && lines(a.residual, a.residual_stride, size) &&
                      uint64_t(a.rows) * a.cols * size * (a.residual ? 2u : 1u) >= kInputsPast;
    return with_type(a.dtype, [&](auto of) {
        using T = decltype(of);
        if constexpr (sizeof(T) == 2)
            if (once) { hipLaunchKernelGGL((k_dropout<T, true>), grid, wg, 0, s, a); return; }
        hipLaunchKernelGGL((k_dropout<T, false>), grid, wg, 0, s, a);
    });
}

// 8 values to a thread, of columns whose sums it keeps.
static uint32_t backward_threads(uint32_t cols)
{
    uint32_t threads = 8;
    while (threads < 1024u && threads * 8u < cols) threads *= 2u;
    return threads;
}

uint32_t norm_parts(uint64_t rows, uint32_t cols)
{
    const uint32_t teams = kBackThreads / backward_threads(cols);
    return uint32_t(std::min<uint64_t>((rows + teams - 1u) / teams, kComputeUnits));
}

// Calls f with what goes past the caches; inputs: so many tensors of `values` values, whole lines of them or not.
template <typename T, typename F> static void with_flow(uint64_t values, uint32_t inputs, bool whole_lines, F &&f)
{
    if constexpr (sizeof(T) == 4) {
        if (values > uint64_t(16) << 20) return f(std::integral_constant<int, CACHED>());
    } else if (whole_lines && values * sizeof(T) * inputs >= kInputsPast) return f(std::integral_constant<int, ALL_PAST>());
    f(std::integral_constant<int, RESULTS_PAST>());
}

// Calls f with the number of threads.
template <typename F> static void with_threads(uint32_t threads, F &&f)
{
    switch (threads) {
    case 8: return f(std::integral_constant<int, 8>());
    case 16: return f(std::integral_constant<int, 16>());
    case 32: return f(std::integral_constant<int, 32>());
    case 64: return f(std::integral_constant<int, 64>());
    case 128: return f(std::integral_constant<int, 128>());
    case 256: return f(std::integral_constant<int, 256>());
    case 512: return f(std::integral_constant<int, 512>());
    default: return f(std::integral_constant<int, 1024>());
    }
}

// Idle LDS of a workgroup, to have fewer of them on a compute unit.  Memory serves large calls with a residual best while about 96 KB a
// unit are on their way to it; all that fit would ask for 128 (16 bits) or 256.  All / so many, in us: 16384 x 4096 bf16 105 / 99, f32 203 / 188, 8192 x 8192
// bf16 101 / 97; smaller calls, narrower rows and calls without a residual lose (2000 x 4096 bf16 13.6 / 14.5; 165536 x 300 95 / 106; without 58 / 60).
static uint32_t idle_lds(const NormForward &a, uint32_t size, uint32_t wg)
{
    if (!a.residual || a.cols <= 1024u || uint64_t(a.rows) * a.cols * size * 4u < (uint64_t(256) << 20)) return 0;
    const uint32_t fit = std::max(2u, (96u << 10) / (wg * 2u * 8u * size * 2u));   // two groups of 8 from two tensors to a thread
    return fit * wg >= 2048u ? 0u : (160u << 10) / (fit + 1u) + 256u;
}

int launch_norm_forward(const NormForward &args, uint32_t dtype, void *stream)
{
    const uint32_t threads = norm_forward_threads(args.cols);
    const RowForm form = {threads, 0};
    const uint32_t wg = form.workgroup(), teams = form.teams();
    const uint64_t step = norm_forward_rows(form);
    const uint64_t size = dtype == ADACOMP_DTYPE_F32 ? 4u : 2u;
    for (uint64_t first = 0; first < args.all_rows; first += step) {
        NormForward a = args;
        const auto on = [first, size](const void *p, uint64_t stride) { return p ? static_cast<const char *>(p) + first * stride * size : nullptr; };
        a.first_row = first;
        a.rows = uint32_t(std::min(step, args.all_rows - first));
        a.x = on(a.x, a.x_stride);
        a.residual = on(a.residual, a.residual_stride);
        a.z = const_cast<char *>(on(a.z, a.z_stride));
        a.y = const_cast<char *>(on(a.y, a.y_stride));
        if (a.mean) a.mean += first;
        if (a.rstd) a.rstd += first;
        const dim3 grid((a.rows + teams - 1u) / teams);
        const uint32_t lds = idle_lds(a, uint32_t(size), wg);
        const bool whole_lines = a.cols % 32u == 0u && lines(a.x, a.x_stride, size) && lines(a.residual, a.residual_stride, size);
        hipStream_t s = static_cast<hipStream_t>(stream);
        const int rc = with_type(dtype, [&](auto of) {
            using T = decltype(of);
            with_flow<T>(args.all_rows * a.cols, a.residual ? 2u : 1u, whole_lines, [&](auto flow) {
                constexpr int FLOW = decltype(flow)::value;
                if (a.cols <= 64u) hipLaunchKernelGGL((k_norm_forward<T, 8, 1, FLOW>), grid, dim3(wg), lds, s, a);
                else if (a.cols > 16384u) hipLaunchKernelGGL((k_norm_forward<T, 1024, 4, FLOW>), grid, dim3(wg), lds, s, a);
                else with_threads(threads, [&](auto n) { hipLaunchKernelGGL((k_norm_forward<T, decltype(n)::value, 2, FLOW>), grid, dim3(wg), lds, s, a); });
            });
        });
        if (rc) return rc;
    }
    return ADACOMP_OK;
}

int launch_norm_backward(const NormBackward &a, uint32_t dtype, uint32_t parts, void *stream)
{
    const dim3 grid(parts), wg(kBackThreads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto of) {
        using T = decltype(of);
        if (a.cols > 16384u) { hipLaunchKernelGGL((k_norm_backward_wide<T, 4>), grid, wg, 0, s, a); return; }
        if (a.cols > 8192u) { hipLaunchKernelGGL((k_norm_backward_wide<T, 2>), grid, wg, 0, s, a); return; }
        const bool whole_lines = a.cols % 32u == 0u && lines(a.dy, a.dy_stride, sizeof(T)) && lines(a.z, a.z_stride, sizeof(T)) && lines(a.dz_add, a.dz_add_stride, sizeof(T));
        with_flow<T>(uint64_t(a.rows) * a.cols, a.dz_add ? 3u : 2u, whole_lines, [&](auto flow) {
            constexpr int FLOW = decltype(flow)::value;
            with_threads(backward_threads(a.cols), [&](auto n) { hipLaunchKernelGGL((k_norm_backward<T, decltype(n)::value, FLOW>), grid, wg, 0, s, a); });
        });
    });
}

int launch_norm_reduce(const NormReduce &a, void *stream)
{
    hipLaunchKernelGGL(k_norm_reduce, dim3((a.cols + 31u) / 32u, 2), dim3(1024), 0, static_cast<hipStream_t>(stream), a);
    return check_launch();
}

}  // namespace adacomp
