// k_embed.cu -- rows of a table by token, scaled, and the gradient of the table.
//   forward   y_r = s w[t_r], 0 where t_r is no row of the table
//   backward  dw_v = s sum of dy_r over the rows with t_r = v
//
// Forward: a row of the table on its way to y, bound by memory.
//
// Backward: the rows are sorted by token, so that a token's rows lie together in
// their first order, and summed by tiles of neighbouring places: a group of lanes
// takes a tile, adds up run after run of equal tokens in registers and writes
// those that begin and end in its tile.  What a tile holds of a run that crosses
// its borders goes to the workspace in 32 bits, and a second kernel adds the
// pieces in the order of the tiles.  So a token of half of all rows (the empty
// cell) is summed by as many groups as its rows fill tiles, and sums have one
// order: no atomics on values.  Rows of the table without a token are zeros,
// written beside the sort's first kernel, whose few blocks leave the memory idle.
//
// The sort takes digits of up to nine bits, from the lowest: blocks count their
// digits, and each block finds its places from the counts of all, so no block
// waits for another.  Up to 4,096 rows one block does it all in shared memory.
#include <type_traits>

#include "async.cuh"
#include "rows.cuh"

namespace av {
namespace {

constexpr int kEmbedThreads = 256;

// What a lane reads at once: kP neighbours in packs of 16 bytes, or one value.  Reading and widening are apart, so that
// the reads of several rows are under way together.
template <class T, int kP>
struct Raw {
    static constexpr int kPack = 16 / sizeof(T), kPacks = kP == 1 ? 1 : kP / kPack;
    std::conditional_t<kP == 1, T, uint4> q[kPacks];
    __device__ __forceinline__ void read(const T *p)
    {
        if constexpr (kP == 1) {
            q[0] = *p;
        } else {
#pragma unroll
            for (int c = 0; c < kPacks; ++c)
                q[c] = reinterpret_cast<const uint4 *>(p)[c];
        }
    }
    __device__ __forceinline__ void widen(float (&v)[kP]) const
    {
        const T *t = reinterpret_cast<const T *>(q);
#pragma unroll
        for (int e = 0; e < kP; ++e)
            v[e] = to_f32(t[e]);
    }
};
template <class T, int kP>
__device__ __forceinline__ void put(T *p, const float (&v)[kP])
{
    if constexpr (kP == 1) {
        *p = from_f32<T>(v[0]);
    } else {
        constexpr int kPack = 16 / sizeof(T);
#pragma unroll
        for (int c = 0; c < kP; c += kPack) {
            uint4 q;
            T *t = reinterpret_cast<T *>(&q);
#pragma unroll
            for (int e = 0; e < kPack; ++e)
                t[e] = from_f32<T>(v[c + e]);
            *reinterpret_cast<uint4 *>(p + c) = q;
        }
    }
}

// ------------------------------------------------------------ forward

// kLanes lanes a row, kRows rows each at a time: kP neighbours a lane, or kPer values kLanes apart.  262,144 rows of 256
// 16-bit values from a table of 65,536 32 us, 5.2 TB/s; 100,003 of 321 32-bit ones, value by value, 37 us, 5.2 TB/s.
template <class W, class Y, int kP, int kPer, int kLanes, int kRows>
__global__ __launch_bounds__(kEmbedThreads) void embed_kernel(int64_t rows, int64_t V, int64_t D, float scale,
                                                              const void *tokens, int token_bytes, const W *w, Y *y,
                                                              int64_t ys)
{
    const int lane = threadIdx.x % kLanes;
    const int64_t first = ((int64_t)blockIdx.x * kEmbedThreads + threadIdx.x) / kLanes * kRows;
    int64_t t[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k)
        t[k] = first + k < rows ? token_of(tokens, token_bytes, first + k) : -1;
    bool has[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        has[k] = t[k] >= 0 && t[k] < V;
        t[k] = has[k] ? t[k] : 0;  // (the table has a row)
    }
    for (int64_t c = lane * kP; c < D; c += kLanes * kP * kPer) {
        Raw<W, kP> raw[kRows][kPer];
#pragma unroll
        for (int k = 0; k < kRows; ++k)
#pragma unroll
            for (int q = 0; q < kPer; ++q)
                raw[k][q].read(w + t[k] * D + (kPer == 1 ? c : min(c + q * kLanes * kP, D - kP)));
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            if (first + k >= rows)
                break;
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                if (kPer > 1 && c + q * kLanes * kP >= D)
                    break;
                float v[kP];
                raw[k][q].widen(v);
#pragma unroll
                for (int e = 0; e < kP; ++e)
                    v[e] = has[k] ? v[e] * scale : 0.0f;
                put<Y, kP>(y + (first + k) * ys + c + q * kLanes * kP, v);
            }
        }
    }
}

// ------------------------------------------------------------ sort

constexpr int kDigit = 9;           // bits of a digit at most
constexpr int kBins = 1 << kDigit;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kEach = 4;            // keys a thread
constexpr int kSorted = kSortThreads * kEach;  // keys a block
// Blocks whose counts a block sums by itself, else a kernel does it for all: 20,000 rows (five blocks) 32.7 us and 34.4 with
// the kernel, 100,000 43.1 and 41.9, 262,144 82.7 and 74.8.
constexpr int kInlineBlocks = 16;

// (key, row); the key is the token, or V where it is none.
using Pair = uint2;

// The pairs of places i[k], those past the last as the last's: kFrom is the bytes of a token, or 0 where pairs are there.
template <int kFrom>
__device__ __forceinline__ void read_pairs(const void *tokens, const Pair *in, int64_t V, int64_t rows, const int64_t (&i)[kEach],
                                           Pair (&pair)[kEach])
{
    if constexpr (kFrom == 0) {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            pair[k] = in[min(i[k], rows - 1)];
    } else {
        int64_t t[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            t[k] = token_of(tokens, kFrom, min(i[k], rows - 1));
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            pair[k] = make_uint2((uint32_t)(t[k] >= 0 && t[k] < V ? t[k] : V), (uint32_t)i[k]);
    }
}

// The lanes that have this lane's digit, of those that have one: a ballot a bit (the match instruction takes a turn for
// every digit that the warp holds; 262,144 rows were sorted in 50 us by it).
__device__ __forceinline__ uint32_t same_digit(uint32_t d, bool here)
{
    uint32_t same = __ballot_sync(~0u, here);
#pragma unroll
    for (int b = 0; b < kDigit; ++b) {
        const bool set = d >> b & 1;
        const uint32_t those = __ballot_sync(~0u, set);
        same &= set ? those : ~those;
    }
    return same;
}

struct SortScratch {
    uint16_t of_warps[kSortWarps][kBins];
    uint32_t warp_sums[kSortWarps];
    uint32_t start[kBins];
    uint2 other[kBins];
    uint32_t local[kBins];
};

__device__ __forceinline__ void zero(void *p, int64_t bytes, int64_t part, int64_t parts)
{
    // (tables lie on the alignment of their type: 16 bytes at a time between the first and last boundary)
    uint8_t *b = (uint8_t *)p;
    const int64_t head = min((int64_t)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15), bytes), packs = (bytes - head) / 16;
    const int64_t step = parts * blockDim.x, at = part * blockDim.x + threadIdx.x;
    for (int64_t i = at; i < packs; i += step)
        reinterpret_cast<uint4 *>(b + head)[i] = make_uint4(0, 0, 0, 0);
    for (int64_t i = at; i < bytes - packs * 16; i += step)
        b[i < head ? i : i + packs * 16] = 0;
}

// Places of this thread's keys among equal digits of the block, in the keys' order: rank[k] within the warp and
// digit, and of_warps turned into what the warps before hold.  Threads hold keys thread-strided within a warp's
// kEach * 32; here[k]: whether there is a k-th.  Returns the block's count of digit threadIdx.x (0 of threads past them).
__device__ uint32_t rank_digits(SortScratch &s, const uint32_t (&digit)[kEach], const bool (&here)[kEach],
                                uint32_t (&rank)[kEach])
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int b = lane; b < kBins; b += 32)
        s.of_warps[warp][b] = 0;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const uint32_t same = same_digit(digit[k], here[k]), before = same & ((1u << lane) - 1);
        const uint32_t held = s.of_warps[warp][digit[k]];
        rank[k] = held + __popc(before);
        __syncwarp();
        if (here[k] && before == 0)
            s.of_warps[warp][digit[k]] = (uint16_t)(held + __popc(same));
        __syncwarp();
    }
    __syncthreads();
    uint32_t sum = 0;
    if (threadIdx.x < kBins) {
#pragma unroll 8
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t n = s.of_warps[w][threadIdx.x];
            s.of_warps[w][threadIdx.x] = (uint16_t)sum;
            sum += n;
        }
    }
    return sum;
}

// The sum of the threads' values before this one's.
__device__ uint32_t before_me(SortScratch &s, uint32_t v)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t sum = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const uint32_t u = __shfl_up_sync(~0u, sum, o);
        sum += lane >= o ? u : 0;
    }
    if (lane == 31)
        s.warp_sums[warp] = sum;
    __syncthreads();
    const uint32_t others = s.warp_sums[lane];
    return __reduce_add_sync(~0u, lane < warp ? others : 0) + sum - v;
}

static_assert(2 * kBins == kSortThreads && kSortWarps == 32, "two threads a digit, a lane a warp");

// All rows in one block; blocks after the first zero the table's gradient.  4,096 rows of 256 values, with what follows,
// 18.7 us, and 27.1 by the kernels for more.
template <int kFrom>
__global__ __launch_bounds__(kSortThreads) void embed_sort_small_kernel(int rows, int64_t V, int bits, int passes,
                                                                        const void *tokens, Pair *out, void *dw, int64_t dw_bytes)
{
    extern __shared__ Pair held[];  // [kSorted]
    __shared__ SortScratch s;
    next_may_start();
    if (blockIdx.x > 0) {
        zero(dw, dw_bytes, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Pair pair[kEach];
    int64_t at[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        at[k] = (warp * kEach + k) * 32 + lane;
    read_pairs<kFrom>(tokens, nullptr, V, rows, at, pair);
    for (int p = 0; p < passes; ++p) {
        uint32_t digit[kEach], rank[kEach];
        bool here[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            here[k] = at[k] < rows;
            digit[k] = pair[k].x >> (p * bits) & ((1u << bits) - 1);
        }
        const uint32_t count = rank_digits(s, digit, here, rank);
        const uint32_t start = before_me(s, count);
        if (threadIdx.x < kBins)
            s.start[threadIdx.x] = start;
        __syncthreads();
        // (the last pass leaves the places in memory, the others in shared memory)
        Pair *to = p == passes - 1 ? out : held;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (here[k])
                to[s.start[digit[k]] + s.of_warps[warp][digit[k]] + rank[k]] = pair[k];
        __syncthreads();
        if (p < passes - 1) {
#pragma unroll
            for (int k = 0; k < kEach; ++k)
                pair[k] = held[at[k] < rows ? at[k] : 0];
            __syncthreads();
        }
    }
}

// counts[block][digit]; blocks after the counting ones zero the table's gradient (first pass).  262,144 rows are sorted by
// two digits in some 35 us (9 + 4 + 8 and 5 + 4 + 8): 64 SMs at work, a chain of short kernels.
template <int kFrom>
__global__ __launch_bounds__(kSortThreads) void embed_count_kernel(int64_t rows, int64_t V, int shift, int bits,
                                                                   const void *tokens, const Pair *in, uint32_t *counts, int blocks,
                                                                   void *dw, int64_t dw_bytes)
{
    __shared__ uint32_t bins[kBins];
    next_may_start();
    if ((int)blockIdx.x >= blocks) {
        zero(dw, dw_bytes, blockIdx.x - blocks, gridDim.x - blocks);
        return;
    }
    const int lane = threadIdx.x & 31;
    if (threadIdx.x < kBins)
        bins[threadIdx.x] = 0;
    __syncthreads();
    if (kFrom == 0)
        after_previous();
    Pair pair[kEach];
    int64_t at[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        at[k] = (int64_t)blockIdx.x * kSorted + k * kSortThreads + threadIdx.x;
    read_pairs<kFrom>(tokens, in, V, rows, at, pair);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const uint32_t d = pair[k].x >> shift & ((1u << bits) - 1), same = same_digit(d, at[k] < rows);
        if (at[k] < rows && (same & ((1u << lane) - 1)) == 0)
            atomicAdd(&bins[d], __popc(same));
    }
    __syncthreads();
    if (threadIdx.x < kBins)
        counts[(int64_t)blockIdx.x * kBins + threadIdx.x] = bins[threadIdx.x];
}

// Of many blocks: counts turned into the sums of the blocks before, the totals behind the last block's.
__global__ __launch_bounds__(1024) void embed_sums_kernel(uint32_t *counts, int blocks)
{
    __shared__ uint32_t parts[32][33];
    next_may_start();
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t *column = counts + blockIdx.x * 32 + lane;
    const int b0 = (int)((int64_t)blocks * warp / 32), b1 = (int)((int64_t)blocks * (warp + 1) / 32);
    uint32_t sum = 0;
    for (int b = b0; b < b1; ++b)
        sum += column[(int64_t)b * kBins];
    parts[warp][lane] = sum;
    __syncthreads();
    uint32_t base = 0;
    for (int k = 0; k < warp; ++k)
        base += parts[k][lane];
    for (int b = b0; b < b1; ++b) {
        const uint32_t n = column[(int64_t)b * kBins];
        column[(int64_t)b * kBins] = base;
        base += n;
    }
    if (warp == 31)
        column[(int64_t)blocks * kBins] = base;
}

// Pairs to their places by one digit, by way of shared memory, where those of a digit come to lie side by side, so that
// neighbouring threads write neighbouring places.
template <int kFrom>
__global__ __launch_bounds__(kSortThreads) void embed_scatter_kernel(int64_t rows, int64_t V, int shift, int bits,
                                                                     const void *tokens, const Pair *in, const uint32_t *counts,
                                                                     int blocks, bool summed, Pair *out)
{
    extern __shared__ Pair held[];  // [kSorted]
    __shared__ SortScratch s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, me = blockIdx.x;
    next_may_start();
    if (kFrom == 0)  // (tokens were there before the call)
        after_previous();
    Pair pair[kEach];
    uint32_t digit[kEach], rank[kEach];
    bool here[kEach];
    int64_t at[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        at[k] = (int64_t)me * kSorted + (warp * kEach + k) * 32 + lane;
    read_pairs<kFrom>(tokens, in, V, rows, at, pair);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        here[k] = at[k] < rows;
        digit[k] = pair[k].x >> shift & ((1u << bits) - 1);
    }
    const uint32_t count = rank_digits(s, digit, here, rank), local = before_me(s, count);
    if (threadIdx.x < kBins)
        s.local[threadIdx.x] = local;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        if (here[k])
            held[s.local[digit[k]] + s.of_warps[warp][digit[k]] + rank[k]] = pair[k];
    if (kFrom != 0)
        after_previous();
    // of a digit: how many the blocks before hold, and all; two threads add up every other block's
    const int bin = threadIdx.x & (kBins - 1), half = threadIdx.x / kBins;
    uint32_t mine = 0, total = 0;
    if (summed) {
        if (half == 0) {
            mine = counts[(int64_t)me * kBins + bin];
            total = counts[(int64_t)blocks * kBins + bin];
        }
    } else {
        constexpr int kAhead = 16;
        for (int b0 = half; b0 < blocks; b0 += 2 * kAhead) {
            uint32_t n[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                n[u] = counts[min(b0 + 2 * u, blocks - 1) * kBins + bin];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                mine += b0 + 2 * u < me ? n[u] : 0;
                total += b0 + 2 * u < blocks ? n[u] : 0;
            }
        }
        if (half == 1)
            s.other[bin] = make_uint2(mine, total);
        __syncthreads();
        if (half == 0) {
            mine += s.other[bin].x;
            total += s.other[bin].y;
        }
    }
    const uint32_t start = before_me(s, half == 0 ? total : 0) + mine;
    if (half == 0)
        s.start[bin] = start - s.local[bin];
    __syncthreads();
    const int n = (int)min((int64_t)kSorted, rows - (int64_t)me * kSorted);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const int i = k * kSortThreads + threadIdx.x;
        if (i < n)
            out[s.start[held[i].x >> shift & ((1u << bits) - 1)] + i] = held[i];
    }
}

// ------------------------------------------------------------ sums

constexpr int kAheadRows = 8;  // rows under way; tiles are multiples of it
constexpr uint32_t kNone = 0xffffffffu;  // no key

// kLanes lanes a tile of `span` places and a part of the columns: kP neighbours a lane, or kPer of them kLanes apart.
// 262,144 rows of 256 16-bit values 33 us, 4.0 TB/s of dy, 60 instructions a row, half of the issue slots.
template <class Y, class W, int kP, int kPer, int kLanes>
__global__ __launch_bounds__(kEmbedThreads, 3) void embed_tiles_kernel(int64_t rows, int64_t V, int64_t D, float scale, int span,
                                                                    const Pair *pairs, const Y *dy, int64_t ys, W *dw,
                                                                    float *parts)
{
    constexpr int kCols = kP * kPer, kAhead = kLanes < 8 || kPer > 1 ? kAheadRows / 2 : kAheadRows;
    const int lane = threadIdx.x % kLanes;
    const int64_t tile = ((int64_t)blockIdx.x * kEmbedThreads + threadIdx.x) / kLanes, i0 = tile * span;
    const int64_t c0 = (int64_t)blockIdx.y * kLanes * kCols + lane * kP;
    next_may_start();
    after_previous();
    if (i0 >= rows)
        return;
    const int n = (int)min((int64_t)span, rows - i0);  // places
    pairs += i0;
    const uint32_t before = i0 > 0 ? pairs[-1].x : kNone, after = i0 + n < rows ? pairs[n].x : kNone, words = (uint32_t)V;
    const Y *from[kPer];
#pragma unroll
    for (int q = 0; q < kPer; ++q)  // (columns past the last: read, not used)
        from[q] = dy + min(c0 + q * kLanes * kP, D - kP);
    float acc[kPer][kP];
    uint32_t run = kNone;
    bool opened = false;  // whether the run begins in this tile
    // What is left of the run; `open`: it may go on in the next tile.
    auto close = [&](bool open) {
        if (run >= words)  // (also where there is none yet)
            return;
        const bool goes_on = open && after == run;
        if (opened && !goes_on) {
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                const int64_t c = c0 + q * kLanes * kP;
                if (c < D) {
                    float v[kP];
#pragma unroll
                    for (int e = 0; e < kP; ++e)
                        v[e] = acc[q][e] * scale;
                    put<W, kP>(dw + (int64_t)run * D + c, v);
                }
            }
        } else {
            float *to = parts + (tile * 2 + (opened ? 1 : 0)) * D;
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                const int64_t c = c0 + q * kLanes * kP;
                if (c < D)
                    put<float, kP>(to + c, acc[q]);
            }
        }
    };
    // the pairs, a group's lanes one each: those of the next kLanes places come while these are taken
    const uint32_t group = kLanes == 32 ? ~0u : ((1u << kLanes) - 1) << (threadIdx.x & 31 & ~(kLanes - 1));
    Pair mine{}, next = pairs[min(lane, n - 1)];
    for (int i = 0; i < n; i += kAhead) {
        if (i % kLanes == 0) {
            mine = next;
            next = pairs[min(i + kLanes + lane, n - 1)];
        }
        Pair pair[kAhead];
        Raw<Y, kP> raw[kAhead][kPer];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            pair[u].x = __shfl_sync(group, mine.x, i + u, kLanes);
            pair[u].y = __shfl_sync(group, mine.y, i + u, kLanes);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int q = 0; q < kPer; ++q)  // (also of rows without a token)
                raw[u][q].read(from[q] + pair[u].y * ys);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= n)
                break;
            if (pair[u].x != run) {
                close(false);
                opened = i + u > 0 || pair[u].x != before;
                run = pair[u].x;
#pragma unroll
                for (int q = 0; q < kPer; ++q)
#pragma unroll
                    for (int e = 0; e < kP; ++e)
                        acc[q][e] = 0.0f;
            }
            if (run < words) {
#pragma unroll
                for (int q = 0; q < kPer; ++q) {
                    float v[kP];
                    raw[u][q].widen(v);
                    if constexpr (kP == 1) {
                        acc[q][0] += v[0];
                    } else {
#pragma unroll
                        for (int e = 0; e < kP; e += 2) {
                            const float2 t = add2(make_float2(acc[q][e], acc[q][e + 1]), make_float2(v[e], v[e + 1]));
                            acc[q][e] = t.x;
                            acc[q][e + 1] = t.y;
                        }
                    }
                }
            }
        }
    }
    close(true);
}

constexpr int kJoinThreads = 512;
constexpr int kJoinWarps = kJoinThreads / 32;
constexpr int kJoinTiles = 32;  // tiles whose runs a block looks for
constexpr int kLongRun = 16;    // pieces from which on the whole block takes a run

struct Run {
    int64_t tile;  // where it begins
    int n;         // pieces
    uint32_t key;
};

// Runs that cross tiles, each by the tile where it begins; a lane takes kP columns, a block 32 kP.  13 us where one token
// has 88,000 rows: the chain of reads, of keys, of the run's end and of its pieces, sixteen at a time.
template <class W, int kP>
__global__ __launch_bounds__(kJoinThreads, kP == 1 ? 4 : 2) void embed_join_kernel(int64_t rows, int64_t V, int64_t D, float scale, int span,
                                                                  int64_t tiles, const Pair *pairs, const float *parts, W *dw)
{
    __shared__ Run runs[kJoinTiles];
    __shared__ int count;
    __shared__ float sums[kJoinWarps][kP][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = ((int64_t)blockIdx.y * 32 + lane) * kP, at = min(c, D - kP);
    next_may_start();
    after_previous();
    if (threadIdx.x == 0)
        count = 0;
    __syncthreads();
    // whether a run that crosses a border begins in tile `lane` of the block's
    const int64_t t0 = (int64_t)blockIdx.x * kJoinTiles, t = t0 + lane, end = (t + 1) * span;
    uint32_t key = 0xffffffffu;
    bool begins = false;
    if (t < tiles - 1) {
        key = pairs[end - 1].x;
        begins = key < V && pairs[end].x == key && (t == 0 || pairs[t * span - 1].x != key);
    }
    const uint32_t all = __ballot_sync(~0u, begins);
    // pieces k0 to k1 of a run, in order: the tail of its first tile, the heads of those that follow
    auto add_up = [&](auto ahead, const Run &r, int k0, int k1, float (&sum)[kP]) {
        constexpr int kAhead = ahead.value;
#pragma unroll
        for (int e = 0; e < kP; ++e)
            sum[e] = 0.0f;
        for (int k = k0; k < k1; k += kAhead) {
            Raw<float, kP> raw[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int j = min(k + u, k1 - 1);
                raw[u].read(parts + ((r.tile + j) * 2 + (j == 0 ? 1 : 0)) * D + at);
            }
            asm volatile("" ::: "memory");  // (all of them are under way before the first is used)
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                float v[kP];
                raw[u].widen(v);
#pragma unroll
                for (int e = 0; e < kP; ++e)
                    sum[e] += k + u < k1 ? v[e] : 0.0f;
            }
        }
    };
    auto leave = [&](const Run &r, float (&sum)[kP]) {
#pragma unroll
        for (int e = 0; e < kP; ++e)
            if (c + e < D)
                dw[(int64_t)r.key * D + c + e] = from_f32<W>(sum[e] * scale);
    };
    float sum[kP];
    int nth = 0;
    for (uint32_t left = all; left; left &= left - 1) {
        if (nth++ % kJoinWarps != warp)
            continue;
        const int which = __ffs(left) - 1;
        const uint32_t k = __shfl_sync(~0u, key, which);
        // the first tile after it whose last place is another's: lanes look at the next 32, then at every 32nd of what is left
        int64_t lo = t0 + which + 1, hi = tiles, step = 1;
        while (lo < hi) {
            const int64_t look = lo + lane * step;
            const bool other = look >= hi || pairs[min((look + 1) * span, rows) - 1].x != k;
            const uint32_t others = __ballot_sync(~0u, other);
            const int before = others ? __ffs(others) - 1 : 32;  // tiles looked at that the run fills to the end
            hi = others ? min(hi, lo + before * step) : hi;
            lo += before > 0 ? (before - 1) * step + 1 : 0;
            step = (hi - lo + 31) / 32;
        }
        const Run r{t0 + which, (int)(lo - t0 - which) + (lo < tiles && pairs[lo * span].x == k ? 1 : 0), k};
        if (r.n <= kLongRun) {
            add_up(std::integral_constant<int, 4>(), r, 0, r.n, sum);
            leave(r, sum);
        } else if (lane == 0) {
            runs[atomicAdd(&count, 1)] = r;  // (in any order: each is summed by itself)
        }
    }
    __syncthreads();
    const int n_runs = count;
    for (int i = 0; i < n_runs; ++i) {
        const Run r = runs[i];
        add_up(std::integral_constant<int, 16>(), r, (int)((int64_t)r.n * warp / kJoinWarps), (int)((int64_t)r.n * (warp + 1) / kJoinWarps), sum);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kP; ++e)
            sums[warp][e][lane] = sum[e];
        __syncthreads();
        if (warp == 0) {
            for (int w = 1; w < kJoinWarps; ++w)
#pragma unroll
                for (int e = 0; e < kP; ++e)
                    sum[e] += sums[w][e][lane];
            leave(r, sum);
        }
    }
}

// ------------------------------------------------------------ host

// Calls f with the lanes for rows of n accesses.
template <class F>
void with_group(int64_t n, F f)
{
    using std::integral_constant;
    if (n <= 4)
        f(integral_constant<int, 4>());
    else if (n <= 16)
        f(integral_constant<int, 16>());
    else
        f(integral_constant<int, 32>());
}

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int bits_of(int64_t V)
{
    int bits = 0;
    while (bits < 32 && (V >> bits) != 0)  // (keys go up to V)
        ++bits;
    return bits;
}

// Places a tile: as many as let the groups of all tiles run at once (three blocks of eight warps an SM), or in a few equal
// turns; a multiple of eight, 128 at most.  (262,144 rows of 256 values: 43 us with tiles of 64, whose 512 blocks come for
// 456 places, and 33 with tiles of 72; 30,011 of 2,048 38 and 30.)
int span_of(int64_t rows, int64_t D)
{
    // groups of lanes for a tile, in 32nds of a warp, eight values a lane
    const int64_t lanes = D <= 32 ? 4 : D <= 128 ? 16 : up(D, 256) * 32, places = 152 * 3 * 8 * 32;
    const int64_t turns = up(rows * lanes, places * 128), span = up(up(rows * lanes, places * turns), kAheadRows) * kAheadRows;
    return (int)(span < kAheadRows ? kAheadRows : span);
}

struct Layout {
    int64_t pairs[2], counts, parts, bytes;
    int64_t blocks, tiles;
    int span;
};
Layout layout_of(int64_t rows, int64_t V, int64_t D)
{
    Layout l{};
    auto take = [&](int64_t bytes) {
        const int64_t at = l.bytes;
        l.bytes += up(bytes, 256) * 256;
        return at;
    };
    l.blocks = up(rows, kSorted);
    l.span = span_of(rows, D);
    l.tiles = up(rows, l.span);
    l.pairs[0] = take(rows * (int64_t)sizeof(Pair));
    l.pairs[1] = take(l.blocks > 1 ? rows * (int64_t)sizeof(Pair) : 0);
    l.counts = take(l.blocks > 1 ? (l.blocks + 1) * kBins * 4 : 0);
    l.parts = take(l.tiles * 2 * D * 4);
    return l;
}

constexpr int kZeroBlocks = 152 * 2;

}  // namespace

int64_t embed_work_bytes(int64_t rows, int64_t V, int64_t D) { return rows ? layout_of(rows, V, D).bytes : 0; }

cudaError_t launch_embed(int64_t rows, int64_t V, int64_t D, int w_dtype, int dtype, float scale, const void *tokens,
                         int token_bytes, const void *w, void *y, int64_t y_stride, cudaStream_t st)
{
    with_type(w_dtype, [&](auto wv) {
        using W = decltype(wv);
        with_type(dtype, [&](auto yv) {
            using Y = decltype(yv);
            constexpr int kP = sizeof(W) == 4 && sizeof(Y) == 4 ? 4 : 8;
            const bool packed = D % kP == 0 && on16(w) && on16(y) && (rows <= 1 || y_stride % (16 / sizeof(Y)) == 0);
            auto go = [&](auto p, auto per) {
                with_group(up(D, p.value * per.value), [&](auto lanes) {
                    const int64_t groups = kEmbedThreads / lanes.value;
                    // (one row at a time: 262,144 x 256 take 49 us in place of 32, and 256 the same 4.1)
                    constexpr int kRows = per.value == 1 ? 4 : 2;
                    embed_kernel<W, Y, p.value, per.value, lanes.value, kRows><<<(unsigned)up(rows, groups * kRows), kEmbedThreads, 0, st>>>(
                        rows, V, D, scale, tokens, token_bytes, (const W *)w, (Y *)y, y_stride);
                });
            };
            using std::integral_constant;
            if (packed)
                go(integral_constant<int, kP>(), integral_constant<int, 1>());
            else
                go(integral_constant<int, 1>(), integral_constant<int, 4>());
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_embed_grad(int64_t rows, int64_t V, int64_t D, int dtype, int w_dtype, float scale, const void *tokens,
                              int token_bytes, const void *dy, int64_t dy_stride, void *dw, void *work, cudaStream_t st)
{
    const Layout l = layout_of(rows, V, D);
    char *base = (char *)work;
    Pair *pairs[2] = {reinterpret_cast<Pair *>(base + l.pairs[0]), reinterpret_cast<Pair *>(base + l.pairs[1])};
    uint32_t *counts = reinterpret_cast<uint32_t *>(base + l.counts);
    float *parts = reinterpret_cast<float *>(base + l.parts);
    const int64_t dw_bytes = V * D * (w_dtype == AV_F32 ? 4 : 2);
    const int all = bits_of(V), passes = (int)up(all, kDigit), bits = (int)up(all, passes);
    const int64_t clear = up(dw_bytes, 65536);
    const int zeros = (int)(clear < kZeroBlocks ? clear : kZeroBlocks);
    const Pair *sorted;
    cudaError_t e;
    auto sort = [&](auto from_tokens) {
        constexpr int kFrom = from_tokens.value;
        auto room = [](auto kernel) {
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSorted * (int)sizeof(Pair));
        };
        e = l.blocks == 1 ? room(embed_sort_small_kernel<kFrom>) : room(embed_scatter_kernel<kFrom>);
        if (e == cudaSuccess && l.blocks > 1)
            e = room(embed_scatter_kernel<0>);
        if (e != cudaSuccess)
            return e;
        if (l.blocks == 1) {
            embed_sort_small_kernel<kFrom><<<1 + zeros, kSortThreads, kSorted * sizeof(Pair), st>>>((int)rows, V, bits, passes, tokens,
                                                                                                   pairs[0], dw, dw_bytes);
            sorted = pairs[0];
            return cudaGetLastError();
        }
        const Pair *in = nullptr;
        const int blocks = (int)l.blocks;
        const bool summed = blocks > kInlineBlocks;
        for (int p = 0; p < passes; ++p) {
            Pair *out = pairs[p & 1];
            const int shift = p * bits;
            e = launch_chained(p == 0 ? embed_count_kernel<kFrom> : embed_count_kernel<0>, (unsigned)(blocks + (p == 0 ? zeros : 0)),
                               kSortThreads, 0, st, p > 0, rows, V, shift, bits, tokens, in, counts, blocks, dw, dw_bytes);
            if (e == cudaSuccess && summed)
                e = launch_chained(embed_sums_kernel, kBins / 32, 1024, 0, st, true, counts, blocks);
            if (e == cudaSuccess)
                e = launch_chained(p == 0 ? embed_scatter_kernel<kFrom> : embed_scatter_kernel<0>, (unsigned)blocks, kSortThreads,
                                   kSorted * sizeof(Pair), st, true, rows, V, shift, bits, tokens, in, counts, blocks, summed, out);
            if (e != cudaSuccess)
                return e;
            in = out;
        }
        sorted = in;
        return cudaSuccess;
    };
    using std::integral_constant;
    e = token_bytes == 1   ? sort(integral_constant<int, 1>())
        : token_bytes == 2 ? sort(integral_constant<int, 2>())
        : token_bytes == 4 ? sort(integral_constant<int, 4>())
                           : sort(integral_constant<int, 8>());
    if (e != cudaSuccess)
        return e;
    with_type(dtype, [&](auto yv) {
        using Y = decltype(yv);
        with_type(w_dtype, [&](auto wv) {
            using W = decltype(wv);
            constexpr int kP = sizeof(W) == 4 && sizeof(Y) == 4 ? 4 : 8;
            const bool packed = D % kP == 0 && on16(dw) && on16(dy) && (rows <= 1 || dy_stride % (16 / sizeof(Y)) == 0);
            auto go = [&](auto p, auto per) {
                with_group(up(D, p.value * per.value), [&](auto lanes) {
                    const dim3 grid((unsigned)up(l.tiles, kEmbedThreads / lanes.value),
                                    (unsigned)up(D, lanes.value * p.value * per.value));
                    e = launch_chained(embed_tiles_kernel<Y, W, p.value, per.value, lanes.value>, grid, kEmbedThreads, 0, st,
                                       true, rows, V, D, scale, l.span, sorted, (const Y *)dy, dy_stride, (W *)dw, parts);
                });
            };
            if (packed)
                go(integral_constant<int, kP>(), integral_constant<int, 1>());
            else
                go(integral_constant<int, 1>(), integral_constant<int, 4>());
            if (e != cudaSuccess || l.tiles <= 1)
                return;
            auto join = [&](auto p) {
                e = launch_chained(embed_join_kernel<W, p.value>, dim3((unsigned)up(l.tiles - 1, kJoinTiles), (unsigned)up(D, 32 * p.value)),
                                   kJoinThreads, 0, st, true, rows, V, D, scale, l.span, l.tiles, sorted, parts, (W *)dw);
            };
            if (D % 4 == 0)
                join(integral_constant<int, 4>());
            else
                join(integral_constant<int, 1>());
        });
    });
    return e;
}

}  // namespace av
