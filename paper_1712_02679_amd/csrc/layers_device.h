// layers_device.h -- device code that the kernels of adacomp_layers.h share: groups of 8 values, the generator of dropout,
// sums and maxima over the threads of a row.
#pragma once

#include <hip/hip_runtime.h>

#include "layers_plan.h"

namespace adacomp {

using bf16 = __bf16;
using f16 = _Float16;
typedef float f32x8 __attribute__((ext_vector_type(8)));

// 8 neighbouring values in memory.  The type's alignment is that of one value: rows of odd lengths begin anywhere, and the
// memory pipeline takes 16-byte accesses at any address of a value.
template <typename T> struct Raw;
template <> struct Raw<float> { typedef float vec __attribute__((ext_vector_type(8))); typedef vec at __attribute__((aligned(4))); };
template <> struct Raw<bf16> { typedef bf16 vec __attribute__((ext_vector_type(8))); typedef vec at __attribute__((aligned(2))); };
template <> struct Raw<f16> { typedef f16 vec __attribute__((ext_vector_type(8))); typedef vec at __attribute__((aligned(2))); };
template <typename T> using raw8 = typename Raw<T>::vec;

// The first n of 8 values (n >= 8: all, n <= 0: none), zeros behind them.
template <typename T> __device__ __forceinline__ raw8<T> load8(const T *p, int n)
{
    raw8<T> v = {};
    if (n >= 8) {
        v = *reinterpret_cast<const typename Raw<T>::at *>(p);
    } else if (n > 0) {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < n) v[k] = p[k];
    }
    return v;
}

template <typename T> __device__ __forceinline__ void store8(T *p, int n, f32x8 x)
{
    const raw8<T> v = __builtin_convertvector(x, raw8<T>);
    if (n >= 8) {
        *reinterpret_cast<typename Raw<T>::at *>(p) = v;
    } else if (n > 0) {
#pragma unroll
        for (int k = 0; k < 7; ++k)
            if (k < n) p[k] = v[k];
    }
}

template <typename T> __device__ __forceinline__ f32x8 widen(raw8<T> v) { return __builtin_convertvector(v, f32x8); }

// ---- dropout: Philox-4x32 with 7 rounds ---------------------------------------------------------------------------
// A round takes two 32 x 32 -> 64 bit products, at a quarter of the rate of other instructions; 7 rounds (the least that
// passed the paper's test batteries) for 8 values cost less than the memory traffic of a group, 10 rounds for 4 values
// would not.

struct Drop {
    uint32_t seed_lo, seed_hi, stream_lo, stream_hi, threshold;
    float factor;
};

__device__ __forceinline__ Drop drop_of(const DropArgs &a)
{
    uint64_t stream = uint64_t(a.stream_hi) << 32 | a.stream_lo;
    if (a.on && a.step) stream += *a.step;
    return {a.seed_lo, a.seed_hi, uint32_t(stream), uint32_t(stream >> 32), a.threshold, a.factor};
}

__device__ __forceinline__ f32x8 drop8(f32x8 v, const Drop &d, uint32_t group, uint32_t row)
{
    uint32_t c0 = group, c1 = row, c2 = d.stream_lo, c3 = d.stream_hi, k0 = d.seed_lo, k1 = d.seed_hi;
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = uint64_t(0xD2511F53u) * c0, b = uint64_t(0xCD9E8D57u) * c2;
        c0 = uint32_t(b >> 32) ^ c1 ^ k0;
        c1 = uint32_t(b);
        c2 = uint32_t(a >> 32) ^ c3 ^ k1;
        c3 = uint32_t(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t half = k % 2 ? w[k / 2] >> 16 : w[k / 2] & 0xFFFFu;
        v[k] = half >= d.threshold ? v[k] * d.factor : 0.f;
    }
    return v;
}

// A kernel's form as a type, for the functions that pick a kernel.
template <int TPR, int V> struct FormOf { static constexpr int threads = TPR, groups = V; };

// ---- sums and maxima over the threads of a row --------------------------------------------------------------------

struct Add { static __device__ __forceinline__ float of(float a, float b) { return a + b; } };
struct Max { static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); } };

template <int CTRL> __device__ __forceinline__ float dpp(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}

// Over N neighbouring lanes of a wave, the same result in all of them: lanes swap inside quads, halves and rows of 16, and
// the rows of a wave are read out.
template <typename OP, int N> __device__ __forceinline__ float over_lanes(float x)
{
    static_assert(N == 8 || N == 16 || N == 32 || N == 64, "part of a wave");
    x = OP::of(x, dpp<0xB1>(x));              // quad_perm 1 0 3 2
    x = OP::of(x, dpp<0x4E>(x));              // quad_perm 2 3 0 1
    x = OP::of(x, dpp<0x141>(x));             // row_half_mirror: the other quad of 8 lanes
    if constexpr (N >= 16) x = OP::of(x, dpp<0x140>(x));   // row_mirror
    if constexpr (N == 32) x = OP::of(x, __shfl_xor(x, 16, 32));
    if constexpr (N == 64) {
        const int b = __builtin_bit_cast(int, x);
        auto row = [b](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(b, l)); };
        x = OP::of(OP::of(row(0), row(16)), OP::of(row(32), row(48)));
    }
    return x;
}

// Over the waves of a workgroup: `room` holds a value of each wave.  The caller takes another `room` for the next call and the
// first one again after that: whoever writes it then has seen a barrier that all its readers reached afterwards.
template <typename OP, int WAVES> __device__ __forceinline__ float over_waves(float x, float *room)
{
    if (threadIdx.x % 64u == 0u) room[threadIdx.x / 64u] = x;
    __syncthreads();
    float all = room[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) all = OP::of(all, room[w]);
    return all;
}

}  // namespace adacomp
