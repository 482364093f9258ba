// sequence_embed.hip -- kernels of the embedding (adacomp_sequence.h).
#include "layers_device.h"
#include "sequence_plan.h"

namespace adacomp {

// Token i of the call, vocab where that is none.
__device__ __forceinline__ uint32_t token_at(const EmbedArgs &a, uint64_t i)
{
    const int64_t t = a.index64 ? static_cast<const int64_t *>(a.tokens)[i] : int64_t(static_cast<const int32_t *>(a.tokens)[i]);
    return uint64_t(t) < a.vocab ? uint32_t(t) : a.vocab;
}

// The 8 values from column c on of a row of `cols`, zeros behind its end; an incomplete group reads the row's last 8 values.
template <typename T> __device__ __forceinline__ f32x8 group8(const T *row, uint32_t c, uint32_t cols)
{
    if (c + 8u <= cols) return widen<T>(load8(row + c));
    if (cols < 8u) return widen<T>(load_some(row + c, cols - c));
    return shifted(widen<T>(load8(row + cols - 8u)), 8u - cols % 8u);
}

// ---- forward ------------------------------------------------------------------------------------------------------
// One group of 8 columns to a thread, as in dropout: 8 columns of a row are one counter of the generator.

template <typename T> __global__ __launch_bounds__(256) void k_embed_forward(EmbedArgs a)
{
    const Drop d = drop_of(a.drop);
    const uint32_t g = blockIdx.x * 256u + threadIdx.x;
    if (g >= a.rows * a.groups) return;
    const uint32_t r = g / a.groups, c = (g - r * a.groups) * 8u;
    const uint64_t row = a.first_row + r;
    const uint32_t token = token_at(a, row);
    f32x8 v = 0.f;
    if (token < a.vocab) {
        v = group8(a.table + uint64_t(token) * a.cols, c, a.cols) * a.scale;
        if (a.drop.on) v = drop8(v, d, c / 8u, uint32_t(row));
    }
    T *y = static_cast<T *>(a.rows_of) + row * a.stride + c;
    if (c + 8u <= a.cols) store8(y, v);
    else store_some(y, a.cols - c, v);
}

// ---- backward: places sorted by token -----------------------------------------------------------------------------
// A workgroup owns a range of tokens.  It looks at all tokens of the call and counts those below its range, which says where its
// part of the order begins, and those in it, wave by wave: a wave has a run of neighbouring places.  Then it knows where each
// wave's places of each token go, and the waves look at their run again and put them there in order.  No workgroup waits for
// another, and the order does not depend on which of them comes first.

__global__ __launch_bounds__(kSortThreads) void k_embed_sort(EmbedArgs a)
{
    extern __shared__ uint32_t counts[];   // [range][waves]
    __shared__ uint32_t room[kSortWaves];
    const uint32_t lane = threadIdx.x % 64u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);
    const uint32_t low = blockIdx.x * a.range, n = min(a.range, a.vocab - low);
    for (uint32_t i = threadIdx.x; i < n * kSortWaves; i += kSortThreads) counts[i] = 0;
    __syncthreads();
    const uint32_t run = ((a.rows + kSortThreads - 1u) / kSortThreads) * 64u;   // places of a wave: whole chunks of 64
    const uint32_t begin = min(wave * run, a.rows), end = min(begin + run, a.rows);
    uint32_t below = 0;
    for (uint32_t i = begin + lane; i < end; i += 64u) {
        const uint32_t token = token_at(a, i);
        below += token < low ? 1u : 0u;
        if (token - low < n) atomicAdd(&counts[(token - low) * kSortWaves + wave], 1u);
    }
    for (uint32_t s = 32; s > 0; s /= 2u) below += __shfl_xor(below, s);
    if (lane == 0u) room[wave] = below;
    __syncthreads();
    uint32_t base = 0;
    for (uint32_t w = 0; w < kSortWaves; ++w) base += room[w];
    // counts, token by token and in each wave by wave, become where they begin: the first wave adds them up, 64 tokens at a time
    if (wave == 0u) {
        for (uint32_t t = 0; t < n; t += 64u) {
            uint32_t mine = 0;
            if (t + lane < n)
                for (uint32_t w = 0; w < kSortWaves; ++w) mine += counts[(t + lane) * kSortWaves + w];
            uint32_t upto = mine;
            for (uint32_t s = 1; s < 64u; s *= 2u) {
                const uint32_t other = __shfl_up(upto, s);
                if (lane >= s) upto += other;
            }
            uint32_t at = base + upto - mine;
            base += __shfl(upto, 63);
            if (t + lane < n) {
                a.first[low + t + lane] = at;
                for (uint32_t w = 0; w < kSortWaves; ++w) {
                    const uint32_t c = counts[(t + lane) * kSortWaves + w];
                    counts[(t + lane) * kSortWaves + w] = at;
                    at += c;
                }
            }
        }
        if (lane == 0u && low + n == a.vocab) a.first[a.vocab] = base;
    }
    __syncthreads();
    for (uint32_t i = begin; i < end; i += 64u) {
        const bool here = i + lane < end;
        const uint32_t t = here ? token_at(a, i + lane) - low : n;
        uint64_t left = __ballot(t < n);
        while (left) {   // every token among the 64, lanes in order
            const uint32_t which = __builtin_amdgcn_readlane(t, __builtin_ctzll(left));
            const uint64_t same = __ballot(t == which);
            uint32_t *count = &counts[which * kSortWaves + wave];
            if (t == which) {
                const uint32_t before = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1u));
                const uint32_t at = *count;
                a.order[at + before] = i + lane;
                if (before == 0u) *count = at + __builtin_popcountll(same);
            }
            left &= ~same;
        }
    }
}

// ---- backward: sums -----------------------------------------------------------------------------------------------

template <typename T> __global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs a, uint64_t work, uint32_t slabs)
{
    const Drop d = drop_of(a.drop);
    for (uint64_t i = blockIdx.x; i < work; i += gridDim.x) {
        const uint32_t token = uint32_t(i / slabs), c = (uint32_t(i % slabs) * 256u + threadIdx.x) * 8u;
        if (c >= a.cols) continue;
        const uint32_t begin = a.first[token], end = a.first[token + 1u];
        if (begin == end && a.accumulate) continue;
        f32x8 sum = 0.f;
        for (uint32_t k = begin; k < end; ++k) {
            const uint32_t row = a.order[k];
            f32x8 v = group8(static_cast<const T *>(a.rows_of) + uint64_t(row) * a.stride, c, a.cols);
            if (a.drop.on) v = drop8(v, d, c / 8u, row);
            sum += v;
        }
        sum *= a.scale;
        float *out = a.dtable + uint64_t(token) * a.cols;
        if (a.accumulate) sum += group8(out, c, a.cols);
        if (c + 8u <= a.cols) store8(out + c, sum);
        else store_some(out + c, a.cols - c, sum);
    }
}

// ---- launches -----------------------------------------------------------------------------------------------------

int launch_embed_forward(const EmbedArgs &args, uint32_t dtype, void *stream)
{
    EmbedArgs a = args;
    const uint64_t step = std::max<uint64_t>(1, (uint64_t(1) << 30) / a.groups);   // groups of a launch are counted in 32 bits
    for (uint64_t first = 0; first < args.rows; first += step) {
        a.first_row = first;
        a.rows = uint32_t(std::min<uint64_t>(step, args.rows - first));
        const dim3 grid((a.rows * a.groups + 255u) / 256u);
        const int rc = with_type(dtype, [&](auto of) { hipLaunchKernelGGL((k_embed_forward<decltype(of)>), grid, dim3(256), 0, static_cast<hipStream_t>(stream), a); });
        if (rc) return rc;
    }
    return ADACOMP_OK;
}

int launch_embed_backward(const EmbedArgs &args, uint32_t dtype, void *stream)
{
    EmbedArgs a = args;
    hipStream_t s = static_cast<hipStream_t>(stream);
    a.range = embed_range(a.vocab);
    hipLaunchKernelGGL(k_embed_sort, dim3((a.vocab + a.range - 1u) / a.range), dim3(kSortThreads), a.range * kSortWaves * 4u, s, a);
    if (int rc = check_launch()) return rc;
    const uint32_t slabs = (a.groups + 255u) / 256u;
    const uint64_t work = uint64_t(a.vocab) * slabs;
    const dim3 grid(uint32_t(std::min<uint64_t>(work, 1u << 20)));
    return with_type(dtype, [&](auto of) { hipLaunchKernelGGL((k_embed_sum<decltype(of)>), grid, dim3(256), 0, s, a, work, slabs); });
}

}  // namespace adacomp
