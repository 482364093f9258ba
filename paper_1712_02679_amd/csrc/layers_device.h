// layers_device.h -- device code that the kernels of adacomp_layers.h share: groups of 8 values, the generator of dropout,
// sums and maxima over the threads of a row.
#pragma once

#include <hip/hip_runtime.h>

#include "layers_plan.h"

namespace adacomp {

using bf16 = __bf16;
using f16 = _Float16;
typedef float f32x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = float(1.4426950408889634 - double(kLog2e)), kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();

// 8 neighbouring values in memory.  The type's alignment is that of one value: rows of odd lengths begin anywhere, and the
// memory pipeline takes 16-byte accesses at any address of a value.
template <typename T> struct Raw;
template <> struct Raw<float> { typedef float vec __attribute__((ext_vector_type(8))); typedef vec at __attribute__((aligned(4))); };
template <> struct Raw<bf16> { typedef bf16 vec __attribute__((ext_vector_type(8))); typedef vec at __attribute__((aligned(2))); };
template <> struct Raw<f16> { typedef f16 vec __attribute__((ext_vector_type(8))); typedef vec at __attribute__((aligned(2))); };
template <> struct Raw<uint8_t> { typedef uint8_t vec __attribute__((ext_vector_type(8))); typedef vec at __attribute__((aligned(1))); };
template <typename T> using raw8 = typename Raw<T>::vec;

// Value `at` of a row: a 32-bit offset from an address that the wave shares.
template <typename T> __device__ __forceinline__ T *at(T *row, uint32_t col)
{
    return reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(row) + uint32_t(col * sizeof(T)));
}

template <typename T> __device__ __forceinline__ raw8<T> load8(const T *p) { return *reinterpret_cast<const typename Raw<T>::at *>(p); }
template <typename T> __device__ __forceinline__ raw8<T> narrow(f32x8 x) { return __builtin_convertvector(x, raw8<T>); }
// Past the caches too, for 16-bit inputs that are larger than those and begin and end with a line (otherwise neighbours read a line twice):
// 16384 x 4096 bf16, us: residual sum 68.3 / 63.8, norm 98.2 / 96.0, backward 123.2 / 119.7; backward softmax 4 x 16 x 2048 x 2048 329 / 320;
// but residual sum 2000 x 4096 8.8 / 9.5, dropout 5003 x 5999 22.0 / 23.5.
template <typename T> __device__ __forceinline__ raw8<T> load8_once(const T *p) { return __builtin_nontemporal_load(reinterpret_cast<const typename Raw<T>::at *>(p)); }
template <typename T> __device__ __forceinline__ void store8(T *p, f32x8 x) { *reinterpret_cast<typename Raw<T>::at *>(p) = narrow<T>(x); }
// Past the caches of the XCD, whose contents a kernel's end writes out in any case: for 16-bit values of which a wave stores neighbouring
// ones, where every line is written whole (16384 x 4096 bf16, us: residual sum 70.9 / 68.3, norm 99.8 / 97.0, backward 127.5 / 122.2; softmax
// 4 x 16 x 2048 x 2048 171 / 165, backward 306 / 296).  Two stores for 8 32-bit values, and rows that a part of a wave stores, write halves
// of lines: they lose where memory is what bounds (backward norm f32 255 / 291, backward softmax f32 4 x 16 x 2048 x 2048 579 / 613, bf16 512 x 16 x 100 x 100 153 / 182), and
// 32-bit ones win in calls that the memory-side cache holds (norm f32 6007 x 577 9.7 / 8.8, backward 16.3 / 15.5).
template <typename T> __device__ __forceinline__ void store8_past(T *p, f32x8 x) { __builtin_nontemporal_store(narrow<T>(x), reinterpret_cast<typename Raw<T>::at *>(p)); }

// The first n of 8 values, 0 < n < 8, zeros behind them.
template <typename T> __device__ __forceinline__ raw8<T> load_some(const T *p, uint32_t n)
{
    raw8<T> v = {};
#pragma unroll
    for (uint32_t k = 0; k < 7u; ++k)
        if (k < n) v[k] = p[k];
    return v;
}

template <typename T> __device__ __forceinline__ void store_some(T *p, uint32_t n, f32x8 x)
{
    const raw8<T> v = narrow<T>(x);
#pragma unroll
    for (uint32_t k = 0; k < 7u; ++k)
        if (k < n) p[k] = v[k];
}

template <typename T> __device__ __forceinline__ f32x8 widen(raw8<T> v) { return __builtin_convertvector(v, f32x8); }

// x without its first n < 8 values, zeros behind the rest; n is the same for all lanes.
__device__ __forceinline__ f32x8 shifted(f32x8 x, uint32_t n)
{
#pragma unroll
    for (uint32_t step = 1; step < 8u; step *= 2u)
        if (n & step) {
#pragma unroll
            for (uint32_t k = 0; k < 8u; ++k) x[k] = k + step < 8u ? x[k + step] : 0.f;
        }
    return x;
}

// The groups of a row that a thread has: group t + v TPR in round v, `cols` columns in all.  A row whose length is no multiple of 8 ends
// with an incomplete group.  Its thread reads the row's last 8 values instead, and moves them into place when it uses them: reading values
// one by one would make the wave wait for them there and then, and with them for everything that is on its way.
// What goes past the caches: nothing, results (store8_past), where a wave stores neighbouring groups, or the inputs as well.
enum Flow { CACHED, RESULTS_PAST, ALL_PAST };
template <typename T> constexpr int kFlow = sizeof(T) == 2 ? RESULTS_PAST : CACHED;

// SHORT: the row may have fewer than 8 values; otherwise it must have 8.
template <typename T, int TPR, int V, int FLOW = kFlow<T>, bool SHORT = TPR == 8> struct RowGroups {
    static constexpr bool kShort = SHORT;
    uint32_t t, cols, first;   // first: column of the part of the row that the threads hold
    __device__ __forceinline__ uint32_t col(int v) const { return first + (t + uint32_t(v) * TPR) * 8u; }
    __device__ __forceinline__ bool whole(int v) const { return col(v) + 8u <= cols; }
    // groups before the incomplete one, in this part
    __device__ __forceinline__ uint32_t before_last() const { return cols / 8u - first / 8u; }
    __device__ __forceinline__ bool ends_in(int v) const { return cols % 8u != 0u && before_last() / TPR == uint32_t(v); }
    __device__ __forceinline__ bool ends_here() const { return before_last() % TPR == t; }
    // round v of the row's values, for columns that the row has
    __device__ __forceinline__ raw8<T> load_round(const T *row, int v) const
    {
        raw8<T> raw = {};
        if constexpr (kShort)
            if (cols < 8u) {
                if (col(v) == 0u) raw = load_some(row, cols);
                return raw;
            }
        if (col(v) < cols) raw = load_whole(at(row, min(col(v), cols - 8u)));
        return raw;
    }
    __device__ __forceinline__ void load(raw8<T> (&raw)[V], const T *row) const
    {
#pragma unroll
        for (int v = 0; v < V; ++v) raw[v] = load_round(row, v);
    }
    // the same for groups that begin below `upto`, anything elsewhere: no branch, what is not wanted is read where the row begins
    __device__ __forceinline__ void load_below(raw8<T> (&raw)[V], const T *row, uint32_t upto) const
    {
        if constexpr (kShort)
            if (cols < 8u) {
                raw[0] = col(0) < upto ? load_some(row, cols) : raw8<T>{};
                return;
            }
#pragma unroll
        for (int v = 0; v < V; ++v) raw[v] = load_whole(at(row, col(v) < upto ? min(col(v), cols - 8u) : 0u));
    }
    // what was loaded for round v, in its place
    __device__ __forceinline__ f32x8 values(const raw8<T> &raw, int v) const
    {
        f32x8 x = widen<T>(raw);
        if (ends_in(v) && !(kShort && cols < 8u)) {
            const f32x8 y = shifted(x, 8u - cols % 8u);
            if (ends_here()) x = y;
        }
        return x;
    }
    static __device__ __forceinline__ void store_whole(T *p, f32x8 x)
    {
        if constexpr (TPR >= 64 && FLOW != CACHED) store8_past(p, x);
        else store8(p, x);
    }
    static __device__ __forceinline__ raw8<T> load_whole(const T *p)
    {
        if constexpr (FLOW == ALL_PAST) return load8_once(p);
        else return load8(p);
    }
    __device__ __forceinline__ void store_round(T *row, int v, f32x8 x) const
    {
        if (whole(v)) store_whole(at(row, col(v)), x);
        else if (col(v) < cols) store_some(at(row, col(v)), cols % 8u, x);
    }
    // x(v) of every round, to its place
    template <typename F> __device__ __forceinline__ void store(T *row, F &&x) const
    {
        f32x8 some = {};
        bool mine = false;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (col(v) < cols) {
                const f32x8 y = x(v);
                if (whole(v)) store_whole(at(row, col(v)), y);
                else { some = y; mine = true; }
            }
        }
        if (cols % 8u != 0u && mine) store_some(at(row, cols & ~7u), cols % 8u, some);
    }
};

// A value that the compiler takes for a new one: what is made from it inside a loop is made there.  Otherwise everything about
// a row that its threads and length decide moves in front of the loop over rows, and costs it its registers: scalar ones
// spilled to lanes of a vector register and read back every time.  The norm kernels spill none; the softmax kernels, whose arguments alone
// are 72 words for 106 registers, still do, fewer.
__device__ __forceinline__ uint32_t again_uniform(uint32_t x) { asm volatile("" : "+s"(x)); return x; }
__device__ __forceinline__ uint32_t again(uint32_t x) { asm volatile("" : "+v"(x)); return x; }

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

__device__ __forceinline__ Drop again(const Drop &d)
{
    return {again_uniform(d.seed_lo), again_uniform(d.seed_hi), d.stream_lo, d.stream_hi, d.threshold, d.factor};
}

// The 16-bit numbers of a group's 8 columns, two to a word.
__device__ __forceinline__ void numbers8(uint32_t (&w)[4], const Drop &d, uint32_t group, uint32_t row)
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
    w[0] = c0;
    w[1] = c1;
    w[2] = c2;
    w[3] = c3;
}

// Zeros in place of what is dropped; the factor is left to the caller.
__device__ __forceinline__ f32x8 kept8(f32x8 v, const Drop &d, uint32_t group, uint32_t row)
{
    uint32_t w[4];
    numbers8(w, d, group, row);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint16_t number = uint16_t(k % 2 ? w[k / 2] >> 16 : w[k / 2]);
        v[k] = number >= uint16_t(d.threshold) ? v[k] : 0.f;
    }
    return v;
}

__device__ __forceinline__ f32x8 drop8(f32x8 v, const Drop &d, uint32_t group, uint32_t row)
{
    return kept8(v, d, group, row) * d.factor;
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

// exp(x).  Exponents are in natural units, as in the formulas, so that they are finite wherever scale * score is: in units of log2 the lowest
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

// Which of a workgroup's rows a thread belongs to.
template <int TPR> __device__ __forceinline__ uint32_t team_of()
{
    const uint32_t team = threadIdx.x / TPR;
    if constexpr (TPR >= 64) return __builtin_amdgcn_readfirstlane(team);
    return team;
}

// ---- launches -----------------------------------------------------------------------------------------------------

inline int check_launch() { return hipGetLastError() == hipSuccess ? ADACOMP_OK : ADACOMP_EHIP; }

// Calls f with a type.
template <typename F> inline int with_type(uint32_t dtype, F &&f)
{
    if (dtype == ADACOMP_DTYPE_F32) f(float());
    else if (dtype == ADACOMP_DTYPE_BF16) f(bf16());
    else f(f16());
    return check_launch();
}

}  // namespace adacomp
