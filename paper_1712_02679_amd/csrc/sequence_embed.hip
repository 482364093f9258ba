// sequence_embed.hip -- kernels of the embedding (adacomp_sequence.h).
//
// The lookup reads a 32-bit row of the table for every place (those asked for again come from the caches) and writes y: memory bounds it, 16384 x 4096 bf16
// with dropout, from 32768 rows, 49 us (6.0 TB/s; 55 with results through the caches), 65536 x 512 bf16 20 us (7.1 TB/s).  The gradient reads dy once and writes the whole table: three
// launches, sorting, sums and the joining of what several pieces have of a token.  32768 x 1001 bf16 with dropout over 50000 tokens 72 us on inputs that the
// caches hold, 90 on others (2.9 TB/s); zeros of tokens that do not occur are stored while places are sorted (without that 80).  12800 x 512 f32 over
// 65 tokens 26 us, three chains of dependent accesses of 11, 6 and 9.  131072 x 512 bf16 over 50000 117 us, about half of it sorting, whose work is places
// times ranges.
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
    if (c + 8u <= a.cols && sizeof(T) == 2) store8_past(y, v);
    else if (c + 8u <= a.cols) store8(y, v);
    else store_some(y, a.cols - c, v);
}

// ---- backward: places sorted by token -----------------------------------------------------------------------------
// A workgroup owns a range of tokens.  It looks at all tokens of the call and counts those below its range, which says where its
// part of the order begins, and those in it, wave by wave: a wave has a run of neighbouring places.  Then it knows where each
// wave's places of each token go, and the waves look at their run again and put them there in order.  No workgroup waits for
// another, and the order does not depend on which of them comes first.

// kChunks of 64 tokens are on their way to a wave at once, and stay in its registers if it has no more.
template <uint32_t kChunks> __global__ __launch_bounds__(kSortThreads) void k_embed_sort(EmbedArgs a)
{
    extern __shared__ uint32_t counts[];   // [waves][range]
    __shared__ uint32_t room[2][kSortWaves];   // places below the range and in it, of every wave and of every 64 tokens
    __shared__ uint64_t empty[kSortRange / 64u];
    typedef float zeros4 __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t lane = threadIdx.x % 64u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64u);
    const uint32_t low = blockIdx.x * a.range, n = min(a.range, a.vocab - low);
    for (uint32_t i = threadIdx.x; i < n * kSortWaves; i += kSortThreads) counts[i] = 0;
    const uint32_t run = ((a.rows + kSortThreads - 1u) / kSortThreads) * 64u;   // places of a wave: whole chunks of 64
    const uint32_t begin = min(wave * run, a.rows), end = min(begin + run, a.rows);
    uint32_t tokens[kChunks], *mine = counts + wave * n;
    // no branch around a load: they are on their way together
    auto fetch = [&](uint32_t from) __attribute__((always_inline)) {
        auto of = [&](auto whole) __attribute__((always_inline)) {
            constexpr bool WHOLE = decltype(whole)::value;
            auto at = [&](uint32_t k) { return WHOLE ? from + k * 64u + lane : min(from + k * 64u + lane, a.rows - 1u); };
            if (a.index64) {
#pragma unroll
                for (uint32_t half = 0; half < kChunks; half += 16u) {
                    int64_t raw[16];
#pragma unroll
                    for (uint32_t k = 0; k < 16u; ++k) raw[k] = static_cast<const int64_t *>(a.tokens)[at(half + k)];
#pragma unroll
                    for (uint32_t k = 0; k < 16u; ++k) tokens[half + k] = uint64_t(raw[k]) < a.vocab ? uint32_t(raw[k]) : a.vocab;
                }
            } else {
#pragma unroll
                for (uint32_t k = 0; k < kChunks; ++k) tokens[k] = static_cast<const uint32_t *>(a.tokens)[at(k)];   // those that are none lie behind all ranges
            }
            if constexpr (!WHOLE)
#pragma unroll
                for (uint32_t k = 0; k < kChunks; ++k) tokens[k] = from + k * 64u + lane < end ? tokens[k] : a.vocab;
        };
        if (from + kChunks * 64u <= end) of(std::true_type());
        else of(std::false_type());
    };
    if (begin < end) fetch(begin);
    __syncthreads();
    uint32_t below = 0;
    for (uint32_t from = begin; from < end; from += kChunks * 64u) {
        if (from != begin) fetch(from);
#pragma unroll
        for (uint32_t k = 0; k < kChunks; ++k) {
            below += uint32_t(__builtin_popcountll(__ballot(tokens[k] < low)));   // of the wave
            if (tokens[k] - low < n) atomicAdd(&mine[tokens[k] - low], 1u);
        }
    }
    if (lane == 0u) room[0][wave] = below;
    __syncthreads();
    // counts, token by token and in each wave by wave, become where they begin: a token to a thread
    static_assert(kSortRange <= kSortThreads, "a thread for every token");
    const uint32_t token = threadIdx.x;
    uint32_t of_wave[kSortWaves], all = 0;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) {
        of_wave[w] = token < n ? counts[w * n + token] : 0u;
        all += of_wave[w];
    }
    uint32_t upto = all;
    for (uint32_t s = 1; s < 64u; s *= 2u) {
        const uint32_t other = __shfl_up(upto, s);
        if (lane >= s) upto += other;
    }
    if (lane == 63u) room[1][wave] = upto;
    __syncthreads();
    uint32_t at = upto - all, total = 0;
#pragma unroll
    for (uint32_t w = 0; w < kSortWaves; ++w) {
        at += room[0][w] + (w < wave ? room[1][w] : 0u);
        total += room[0][w] + room[1][w];
    }
    if (token < n) {
        a.first[low + token] = at;
#pragma unroll
        for (uint32_t w = 0; w < kSortWaves; ++w) {
            counts[w * n + token] = at;
            at += of_wave[w];
        }
    }
    if (threadIdx.x == 0u && low + n == a.vocab) a.first[a.vocab] = total;
    const uint64_t none = __ballot(token < n && all == 0u);   // of the wave's 64 tokens
    if (lane == 0u && wave < kSortRange / 64u) empty[wave] = none;
    __syncthreads();
    // zeros for the tokens that do not occur: stores that are on their way while the places are put in order
    if (!a.accumulate) {
        const uint32_t beside = 64u / a.zero_team, c = lane % a.zero_team * 4u;   // rows of a wave side by side, 4 columns to a thread
        for (uint32_t t = wave * beside + lane / a.zero_team; t < n; t += kSortWaves * beside) {
            if (!(empty[t / 64u] >> t % 64u & 1u)) continue;
            float *out = a.dtable + uint64_t(low + t) * a.cols;
            for (uint32_t col = c; col < a.cols; col += a.zero_team * 4u) {
                if (col + 4u <= a.cols) *reinterpret_cast<zeros4 *>(out + col) = zeros4(0.f);
                else
                    for (uint32_t k = col; k < a.cols; ++k) out[k] = 0.f;
            }
        }
    }
    for (uint32_t from = begin; from < end; from += kChunks * 64u) {
        if (run > kChunks * 64u) fetch(from);
#pragma unroll
        for (uint32_t k = 0; k < kChunks; ++k) {
            const uint32_t t = tokens[k] - low;
            uint64_t left = __ballot(t < n);
            while (left) {   // every token among the 64, lanes in order
                const uint32_t which = __builtin_amdgcn_readlane(t, __builtin_ctzll(left));
                const uint64_t same = __ballot(t == which);
                volatile uint32_t *count = &mine[which];
                if (t == which) {
                    const uint32_t before = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1u));
                    const uint32_t at = *count;
                    a.order[at + before] = {low + t, from + k * 64u + lane};
                    if (before == 0u) *count = at + __builtin_popcountll(same);
                }
                left &= ~same;
            }
        }
    }
}

// ---- backward: sums -----------------------------------------------------------------------------------------------
// The order is cut into pieces of as many places, whatever their tokens are, so that a frequent token's are shared out like all others.  A team of
// threads has a piece and a slab of columns, 8 to a thread, and adds up the rows of a token while it lasts.  A token whose places lie in
// one piece is done then.  Of one that goes on in another piece every piece leaves its part, and k_embed_join adds them up in order.

constexpr uint32_t kSumThreads = 256;

template <typename T, bool DROP> __global__ __launch_bounds__(kSumThreads) void k_embed_sum(EmbedArgs a)
{
    extern __shared__ EmbedPlace staged[];   // [teams][piece + 2]: the places of a piece, one before and one behind
    constexpr uint32_t BATCH = 16u / sizeof(T);   // rows on their way at once
    const uint32_t t = threadIdx.x & (a.team - 1u), team = threadIdx.x / a.team, teams = kSumThreads / a.team;
    const Drop d = drop_of(a.drop);
    const uint32_t job = blockIdx.x * teams + team, piece = job / a.slabs, slab = job - piece * a.slabs;
    const uint32_t count_all = a.first[a.vocab], begin = min(piece, a.pieces) * a.piece;
    const uint32_t count = begin < count_all && piece < a.pieces ? min(a.piece, count_all - begin) : 0u;
    EmbedPlace *mine = staged + team * (a.piece + 2u);
    for (uint32_t k = t; k < count + 2u; k += a.team) {   // places that there are not hold no token
        const uint32_t at = begin + k;
        mine[k] = at >= 1u && at <= count_all ? a.order[at - 1u] : EmbedPlace{a.vocab, 0u};
    }
    __syncthreads();
    const uint32_t c = (slab * a.team + t) * 8u;
    if (c >= a.cols) return;
    const uint32_t cut = a.cols >= 8u && c + 8u > a.cols ? 8u - a.cols % 8u : 0u;   // an incomplete group reads the row's last 8 values
    const T *dy = static_cast<const T *>(a.rows_of) + (c - cut);
    const uint32_t whole_row = a.cols >= 8u;
    f32x8 sum = 0.f;
    uint32_t run = 0;   // where the token's run begins
    for (uint32_t from = 0; from < count; from += BATCH) {
        raw8<T> raw[BATCH];
#pragma unroll
        for (uint32_t k = 0; k < BATCH; ++k) {
            const T *row = dy + uint64_t(mine[min(from + k, count - 1u) + 1u].row) * a.stride;
            raw[k] = whole_row ? load8(row) : load_some(row, a.cols);
        }
#pragma unroll
        for (uint32_t k = 0; k < BATCH; ++k) {
            const uint32_t at = from + k;
            if (at >= count) break;
            const EmbedPlace place = mine[at + 1u];
            f32x8 v = widen<T>(raw[k]);
            if constexpr (DROP) {
                if (cut) v = shifted(v, cut);
                v = drop8(v, d, c / 8u, place.row);
            }
            sum += v;
            const uint32_t next = mine[at + 2u].token;
            if (next == place.token && at + 1u < count) continue;
            if (!DROP && cut) sum = shifted(sum, cut);
            const bool goes_on = next == place.token, came = run == 0u && mine[0].token == place.token;
            const uint32_t n = a.cols - c;
            if (came || goes_on) {   // a part: behind others, or the first of them
                float *out = a.parts + (uint64_t(piece) * 2u + (came ? 0u : 1u)) * a.pitch + c;
                store8(out, sum);
            } else {
                float *out = a.dtable + uint64_t(place.token) * a.cols + c;
                sum *= a.scale;
                if (a.accumulate) sum += n >= 8u ? widen<float>(load8(out)) : widen<float>(load_some(out, n));
                if (n >= 8u) store8(out, sum);
                else store_some(out, n, sum);
            }
            sum = 0.f;
            run = at + 1u;
        }
    }
}

// Tokens whose places lie in several pieces: their parts, in order.  A workgroup has the tokens of a sorting workgroup and 256 columns, 8 to each of
// 32 threads; of a token with many parts each of its 16 slices of threads takes every 16th, tokens of few parts are the slices' own.
constexpr uint32_t kJoinSlices = 16, kFewParts = 8;

__global__ __launch_bounds__(32 * kJoinSlices) void k_embed_join(EmbedArgs a)
{
    __shared__ f32x8 sums[kJoinSlices][32];
    __shared__ uint32_t list[2][kSortRange], count[2];   // tokens of few parts, of many
    const uint32_t lane = threadIdx.x % 32u, slice = threadIdx.x / 32u, c = (blockIdx.y * 32u + lane) * 8u, n = a.cols - c;
    const uint32_t low = blockIdx.x * a.range, tokens = min(a.range, a.vocab - low);
    if (threadIdx.x < 2u) count[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < tokens; i += 32u * kJoinSlices) {
        const uint32_t begin = a.first[low + i], end = a.first[low + i + 1u];
        if (begin == end || begin / a.piece == (end - 1u) / a.piece) continue;
        const uint32_t many = (end - 1u) / a.piece - begin / a.piece >= kFewParts;
        list[many][atomicAdd(&count[many], 1u)] = low + i;   // in any order: tokens have nothing to do with each other
    }
    __syncthreads();
    const bool live = c < a.cols;
    auto part = [&](uint32_t p, uint32_t begin) {   // the first part of a token lies behind its piece's others
        return widen<float>(load8(a.parts + (uint64_t(p) * 2u + (p == begin ? 1u : 0u)) * a.pitch + c));
    };
    auto put = [&](uint32_t token, f32x8 s) {
        s *= a.scale;
        float *out = a.dtable + uint64_t(token) * a.cols + c;
        if (a.accumulate) s += n >= 8u ? widen<float>(load8(out)) : widen<float>(load_some(out, n));
        if (n >= 8u) store8(out, s);
        else store_some(out, n, s);
    };
    if (live)
        for (uint32_t i = slice; i < count[0]; i += kJoinSlices) {
            const uint32_t token = list[0][i], begin = a.first[token] / a.piece, last = (a.first[token + 1u] - 1u) / a.piece;
            f32x8 s = part(begin, begin);
#pragma unroll 4
            for (uint32_t p = begin + 1u; p <= last; ++p) s += part(p, begin);
            put(token, s);
        }
    for (uint32_t i = 0; i < count[1]; ++i) {
        const uint32_t token = list[1][i], begin = a.first[token] / a.piece, last = (a.first[token + 1u] - 1u) / a.piece;
        f32x8 s = 0.f;
        if (live)
#pragma unroll 8
            for (uint32_t p = begin + slice; p <= last; p += kJoinSlices) s += part(p, begin);
        sums[slice][lane] = s;
        __syncthreads();
        if (slice == 0u && live) {
            for (uint32_t k = 1; k < kJoinSlices; ++k) s += sums[k][lane];
            put(token, s);
        }
        __syncthreads();   // the sums have been read
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
    const EmbedForm form = embed_form(a.rows, a.vocab, a.cols);
    a.range = form.range;
    a.team = form.team;
    a.slabs = form.slabs;
    a.piece = form.piece;
    a.pieces = form.pieces;
    a.pitch = form.pitch;
    a.zero_team = 4;
    while (a.zero_team < 64u && a.zero_team * 4u < a.cols) a.zero_team *= 2u;
    const dim3 ranges((a.vocab + a.range - 1u) / a.range);
    const uint32_t counts = a.range * kSortWaves * 4u;
    if (a.rows <= 16u * kSortThreads) hipLaunchKernelGGL(k_embed_sort<16>, ranges, dim3(kSortThreads), counts, s, a);
    else hipLaunchKernelGGL(k_embed_sort<32>, ranges, dim3(kSortThreads), counts, s, a);
    if (int rc = check_launch()) return rc;
    const uint32_t teams = kSumThreads / a.team;
    const uint32_t blocks = uint32_t((uint64_t(a.pieces) * a.slabs + teams - 1u) / teams);
    if (blocks != 0u) {
        const dim3 grid(blocks), wg(kSumThreads);
        const uint32_t lds = teams * (a.piece + 2u) * 8u;
        const int rc = with_type(dtype, [&](auto of) {
            using T = decltype(of);
            if (a.drop.on) hipLaunchKernelGGL((k_embed_sum<T, true>), grid, wg, lds, s, a);
            else hipLaunchKernelGGL((k_embed_sum<T, false>), grid, wg, lds, s, a);
        });
        if (rc) return rc;
    }
    if (a.pieces < 2u) return ADACOMP_OK;
    hipLaunchKernelGGL(k_embed_join, dim3((a.vocab + a.range - 1u) / a.range, (a.groups + 31u) / 32u), dim3(32u * kJoinSlices), 0, s, a);
    return check_launch();
}

}  // namespace adacomp
