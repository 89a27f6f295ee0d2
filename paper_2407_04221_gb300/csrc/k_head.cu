// k_head.cu -- log probabilities of tokens under the softmax of x w^T, and the
// gradients of x and w, without the logits.
//   l = x w^T,  m = max l,  logz = log sum exp(l - m),  log p_t = (l_t - m) - logz
//   G_rj = dlogp_r (1[j = t_r] - exp((l_rj - m_r) - logz_r)),  dx = G w,  dw = G^T x
//
// The products run on the tensor cores (tcgen05, accumulators in TMEM), a pair of
// CTAs on a tile of 256 rows x 256 words.  Forward, a tile of logits never leaves
// the chip: each row's maximum and sum of exponentials over the tile's words do,
// 8 bytes a row and tile, and a second kernel joins them.  Backward the table is
// taken in pieces of words: the logits of a piece are made again and G of it goes
// to the workspace (the logits whole would be 2 GB at 8,192 x 65,536), from where
// two products take it: dw of the piece, and what the piece adds to dx, summed in
// 32 bits over the pieces.  G goes as two values of 16 bits, the rounded one and
// what that leaves, and sums of 512 terms are added in 32 bits, as those of 256 are
// of the logits, so that only dx and dw are rounded: 10 N V D operations where
// one value would take 6, and the error of rounding once in place of 1.41 times
// it.  float16 has not the range for G: it goes times a power of two, from the
// largest |dlogp|, and the results are brought back before they are rounded.
//
// Rows without a token are not looked at: the others are packed first (x as it is
// where all have one), so a padded batch costs what its tokens cost, and what
// padding holds reaches nothing.
#include "policy.h"
#include "rows.cuh"
#include "tensor.cuh"

namespace av {
namespace {

template <class T>
constexpr bool kScaled = std::is_same<T, __half>::value;

// ------------------------------------------------------------ rows with a token

constexpr int kRowsThreads = 1024;
constexpr int kRowsEach = 8;   // rows of a thread under way

// What the kernels of a call share: the number of rows with a token and the power of two that G goes times.
struct Shared {
    int count;
    float scale;
};

// A row's token and what its gradient takes: its slope is up (1[j = token] - exp((l - m) - z)).
struct Slope {
    float m, z, up;
    int token;
};

// 1 - exp(d).  Where that is small, by the series of (exp(d) - 1) / d, good to 0.5^10 / 11!; 8,192 x 256 x 32,768 with
// the library's function 662 us, so 646.
__device__ __forceinline__ float one_less_exp(float d)
{
    constexpr float kSeries[] = {1.0f / 3628800, 1.0f / 362880, 1.0f / 40320, 1.0f / 5040, 1.0f / 720, 1.0f / 120, 1.0f / 24, 1.0f / 6, 0.5f, 1.0f};
    float sum = 0.0f;
#pragma unroll
    for (float c : kSeries)
        sum = fmaf(sum, d, c);
    return fabsf(d) < 0.5f ? -d * sum : 1.0f - exp2_fast(d * kLog2e);
}

// What brings the largest |G|, which is at most |dlogp|, below 2^15.
__device__ __forceinline__ float scale_for(float top)
{
    if (!(top > 0.0f))
        return 1.0f;
    const int k = 15 - ((int)(__float_as_uint(top) >> 23) - 126);
    return __int_as_float((127 + min(max(k, -100), 100)) << 23);
}

// One block: order[i] is the i-th row that has a token, place[r] where row r went (-1: it has none), tokens[i] its
// token.  Forward: results of rows without one.  Backward (kGrad): slopes.
template <bool kGrad, bool kScale>
__global__ __launch_bounds__(kRowsThreads) void head_rows_kernel(int rows, int64_t V, const void *given, int token_bytes,
                                                                 int *order, int *place, int *tokens, Shared *shared,
                                                                 float *logp, float *peak, float *logz, const float *dlogp,
                                                                 Slope *slopes)
{
    __shared__ int counts[kRowsEach * 32];
    __shared__ int warp_sums[32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    next_may_start();
    float scale = 1.0f;
    if (kScale) {
        float top = 0.0f;
#pragma unroll 8
        for (int r = threadIdx.x; r < rows; r += kRowsThreads) {
            const int64_t t = token_of(given, token_bytes, r);
            const float d = fabsf(dlogp[r]);
            top = t >= 0 && t < V && d <= 3.402823466e38f ? fmaxf(top, d) : top;
        }
        const int most = __reduce_max_sync(~0u, __float_as_int(top));  // (none is negative)
        if (lane == 0)
            warp_sums[warp] = most;
        __syncthreads();
        scale = scale_for(__int_as_float(__reduce_max_sync(~0u, warp_sums[lane])));
        __syncthreads();
    }
    int base = 0;
    for (int64_t r0 = 0; r0 < rows; r0 += kRowsThreads * kRowsEach) {
        int token[kRowsEach];
        uint32_t here[kRowsEach];
#pragma unroll
        for (int k = 0; k < kRowsEach; ++k) {
            const int64_t r = r0 + k * kRowsThreads + threadIdx.x, t = token_of(given, token_bytes, r < rows ? r : 0);
            token[k] = r < rows && t >= 0 && t < V ? (int)t : -1;
        }
#pragma unroll
        for (int k = 0; k < kRowsEach; ++k) {
            here[k] = __ballot_sync(~0u, token[k] >= 0);
            if (lane == 0)
                counts[k * 32 + warp] = __popc(here[k]);
        }
        __syncthreads();
        const int mine = threadIdx.x < kRowsEach * 32 ? counts[threadIdx.x] : 0;
        int to = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int before = __shfl_up_sync(~0u, to, o);
            to += lane >= o ? before : 0;
        }
        if (lane == 31)
            warp_sums[warp] = to;
        __syncthreads();
        const int sum = warp_sums[lane];
        const int before = __reduce_add_sync(~0u, lane < warp ? sum : 0), all = __reduce_add_sync(~0u, sum);
        if (threadIdx.x < kRowsEach * 32)
            counts[threadIdx.x] = before + to - mine;
        __syncthreads();
        float up[kRowsEach], m[kRowsEach], z[kRowsEach];
        if (kGrad) {
#pragma unroll
            for (int k = 0; k < kRowsEach; ++k) {
                const int64_t r = min(r0 + k * kRowsThreads + threadIdx.x, (int64_t)rows - 1);
                up[k] = dlogp[r];
                m[k] = peak[r];
                z[k] = logz[r];
            }
        }
#pragma unroll
        for (int k = 0; k < kRowsEach; ++k) {
            const int64_t r = r0 + k * kRowsThreads + threadIdx.x;
            if (r >= rows)
                break;
            const int i = base + counts[k * 32 + warp] + __popc(here[k] & ((1u << lane) - 1));
            place[r] = token[k] >= 0 ? i : -1;
            if (token[k] >= 0) {
                order[i] = (int)r;
                if (kGrad)
                    slopes[i] = {m[k], z[k], up[k] * scale, token[k]};
                else
                    tokens[i] = token[k];
            } else if (!kGrad) {
                logp[r] = 0.0f;
                if (peak)
                    peak[r] = 0.0f;
                if (logz)
                    logz[r] = 0.0f;
            }
        }
        base += all;
        __syncthreads();
    }
    if (threadIdx.x == 0)
        *shared = {base, scale};
}

// Rows of which every block looks at all tokens.  Forward and back, of 64 columns and 256 words: 16,384 rows 19 and 49 us, in
// two steps 22 and 63; 32,768 31 and 72, and 33 and 101; 65,536 64 and 137, and 56 and 178; 131,072 179 and 310, and 98 and
// 332; 262,144 587 and 830, and 186 and 640.  One number for both passes.
constexpr int kOnceRows = 32768;
constexpr int kOnceThreads = 256;
constexpr int kOnceEach = 64;     // rows of a block

// Both steps in one, of up to kOnceRows rows: each block counts the tokens before its rows and all, so that none waits for
// another, and packs its rows.
template <bool kGrad, bool kScale>
__global__ __launch_bounds__(kOnceThreads) void head_once_kernel(int rows, int64_t V, const void *given, int token_bytes, int *order,
                                                                 int *place, int *tokens, Shared *shared, float *logp, float *peak,
                                                                 float *logz, const float *dlogp, Slope *slopes, int64_t D,
                                                                 const uint4 *x, int64_t xs, uint4 *packed)
{
    constexpr int kWarps = kOnceThreads / 32, kAhead = 16;
    __shared__ int befores[kWarps], alls[kWarps], tops[kWarps], places[kOnceEach];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r0 = blockIdx.x * kOnceEach;
    next_may_start();
    int before = 0, all = 0;
    float top = 0.0f;
    for (int i0 = threadIdx.x; i0 < rows; i0 += kOnceThreads * kAhead) {
        int64_t t[kAhead];
        float d[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = min(i0 + u * kOnceThreads, rows - 1);
            t[u] = token_of(given, token_bytes, i);
            d[u] = kScale ? fabsf(dlogp[i]) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * kOnceThreads;
            const bool has = i < rows && t[u] >= 0 && t[u] < V;
            all += has;
            before += has && i < r0;
            top = kScale && has && d[u] <= 3.402823466e38f ? fmaxf(top, d[u]) : top;
        }
    }
    before = __reduce_add_sync(~0u, before);
    all = __reduce_add_sync(~0u, all);
    const int most = __reduce_max_sync(~0u, __float_as_int(top));  // (none is negative)
    if (lane == 0) {
        befores[warp] = before;
        alls[warp] = all;
        tops[warp] = most;
    }
    __syncthreads();
    before = __reduce_add_sync(~0u, lane < kWarps ? befores[lane] : 0);
    all = __reduce_add_sync(~0u, lane < kWarps ? alls[lane] : 0);
    const float scale = kScale ? scale_for(__int_as_float(__reduce_max_sync(~0u, lane < kWarps ? tops[lane] : 0))) : 1.0f;
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *shared = {all, scale};
    if (warp == 0) {
#pragma unroll
        for (int k = 0; k < kOnceEach / 32; ++k) {
            const int r = r0 + k * 32 + lane, at = min(r, rows - 1);
            const int64_t t = token_of(given, token_bytes, at);
            const bool has = r < rows && t >= 0 && t < V;
            const uint32_t here = __ballot_sync(~0u, has);
            const int i = before + __popc(here & ((1u << lane) - 1));
            before += __popc(here);
            places[k * 32 + lane] = has ? i : -1;
            if (r < rows) {
                place[r] = has ? i : -1;
                if (has) {
                    order[i] = r;
                    if (kGrad)
                        slopes[i] = {peak[r], logz[r], dlogp[r] * scale, (int)t};
                    else
                        tokens[i] = (int)t;
                } else if (!kGrad) {
                    logp[r] = 0.0f;
                    if (peak)
                        peak[r] = 0.0f;
                    if (logz)
                        logz[r] = 0.0f;
                }
            }
        }
    }
    if (all == rows)
        return;
    __syncthreads();
    const int per = (int)(D / 8);
    for (int k = warp; k < kOnceEach; k += kWarps) {
        const int i = places[k];
        if (i >= 0)
            for (int c = lane; c < per; c += 32)
                packed[(int64_t)i * per + c] = __ldg(x + (r0 + k) * (xs / 8) + c);
        const int j = r0 + k;  // of the packed rows, zeros past the last up to the tile's end
        if (j >= all && j < min((int64_t)rows, up(all > 0 ? all : 1, kTile) * kTile))
            for (int c = lane; c < per; c += 32)
                packed[(int64_t)j * per + c] = make_uint4(0, 0, 0, 0);
    }
}

// x's rows with a token side by side, then zeros up to the tile's end; nothing where all rows have one.
__global__ __launch_bounds__(256) void head_pack_kernel(int rows, int64_t D, const uint4 *x, int64_t xs, const int *order,
                                                        const Shared *shared, uint4 *packed)
{
    next_may_start();
    after_previous();
    const int count = shared->count;
    if (count == rows)
        return;
    const int64_t per = D / 8, n = min((int64_t)rows, up(count > 0 ? count : 1, kTile) * kTile) * per;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n; k += (int64_t)gridDim.x * 256) {
        const int64_t i = k / per;
        packed[k] = i < count ? __ldg(x + order[i] * (xs / 8) + k % per) : make_uint4(0, 0, 0, 0);
    }
}

// ------------------------------------------------------------ products

enum Form {
    kStats,      // maxima and sums of a tile's logits
    kSlopes,     // G of a piece, from the logits made again
    kProducts    // of G of a piece: what it adds to dx, G w, where B runs along its rows, and its dw, G^T x, A and B along theirs
};

constexpr int kValues = 2;  // that G goes as: [value][row][word]

__host__ __device__ constexpr bool of_logits(int form) { return form == kStats || form == kSlopes; }
// Fours of warps that take accumulators out; a slab of each; stages of A and B.
__host__ __device__ constexpr int teams_of(int form) { return of_logits(form) ? 4 : 2; }
__host__ __device__ constexpr int slabs_of(int form) { return form == kStats ? 0 : 1; }
__host__ __device__ constexpr int stages_of(int form) { return form == kSlopes ? 5 : 6; }
__host__ __device__ constexpr int threads_of(int form) { return 64 + 128 * teams_of(form); }
__host__ __device__ constexpr int smem_of(int form)
{
    return stages_of(form) * 2 * kHalf + teams_of(form) * slabs_of(form) * kSlab + 1024 + 256 +
           (form == kStats ? 2 * teams_of(form) * kRowsCta * 8 : 0);
}

struct Params {
    int rows;             // of x
    int words;            // of the piece (forward: of the table)
    int first;            // the piece's first word
    int d;                // D
    int dx_splits, dw_splits;  // parts that the terms of a product are dealt to
    bool more;            // dx: there are sums of earlier pieces
    const Shared *shared;
    const int *tokens;    // of the packed rows
    const Slope *slopes;
    float2 *parts;        // [tile of words][row]: maximum, sum
    float *wanted;        // the tokens' logits (backward: those of few rows, summed as forward)
};

// A product's tiles.
struct Work {
    int m_tiles, n_tiles, k_once, k_blocks, splits;
    __device__ __forceinline__ int tiles() const { return m_tiles * n_tiles * splits; }
};

struct Tile {
    int m, n, k0, k1, split;
};

// Blocks of 64 terms that accumulators take before they are added to sums in registers, of logits.  The tensor cores
// truncate at every addition to the accumulator, a bias that grows with their number: of 8,192 x 1,024 x 65,536 the peaks
// are off by 1.1e-6 of themselves, as root mean square, with all terms at once (the call 616 us), by 5.2e-7 with eight blocks
// (632), 2.5e-7 with four (670; sums in 32 bits 3.2e-7) and 1.3e-7 with two (783).  Backward they are the same sums, to the
// last bit: m and logz are of them, and in a row that is sure of its token what is left of one, 1 - p, is of the size of
// such errors (2.5 % of that call's gradient: 3.60 ms with all terms at once, 3.69 with these).
constexpr int kPart = 4;

// The same of the products.  At an addition sixteen products and the sum are truncated, together by some 2^-22.5 of it: sums
// of one sign come out short.  With all terms at once, and with 32, 16, 8 and 4 blocks: dw of 262,144 rows by 8.3e-4, 1.2e-5,
// 5.1e-6, 1.9e-6 and 4e-7 of itself, dx of 100,000 words by 3.5e-4, 1.2e-5, 5.9e-6, 2.8e-6 and 1.3e-6 (float16's largest
// rounding is 4.9e-4); the gradient of 8,192 x 1,024 x 65,536 takes 3.69, 3.80, 3.79, 3.84 and 3.94 ms.
constexpr int kSumPart = 8;
__host__ __device__ constexpr int part_of(int form) { return of_logits(form) ? kPart : kSumPart; }

// Tiles in bands of eight rows of tiles, down the band first: those in flight together share A and B in L2.
__device__ __forceinline__ Tile tile_of(const Work &p, int i)
{
    const int per = p.m_tiles * p.n_tiles;
    Tile t;
    t.split = i / per;
    i -= t.split * per;
    const int band = i / (8 * p.n_tiles), first = band * 8;
    const int high = min(8, p.m_tiles - first);
    const int at = i - band * 8 * p.n_tiles;
    t.m = first + at % high;
    t.n = at / high;
    t.k0 = (int)((int64_t)p.k_blocks * t.split / p.splits);
    t.k1 = (int)((int64_t)p.k_blocks * (t.split + 1) / p.splits);
    return t;
}

// Which tiles a pair takes: the longer product's go round the pairs; of the other's the pairs that came away with one less
// take as many ahead as make up for it, and the rest go round.  How many rows have a token is known on the GPU alone.  The
// gradient of 16,384 x 512 x 32,768 takes 1.97 ms, and 2.25 with both products' tiles going round; of 2,999 x 520 x 50,021, a
// third of the rows without a token, 555 us and 571.
struct Turns {
    int pair, pairs, longer, shorter, rest, ahead;  // tiles; pairs with one more of the longer; tiles taken ahead
    __device__ __forceinline__ Turns(int n_longer, int n_shorter, int long_blocks, int short_blocks)
        : pair(blockIdx.x >> 1), pairs(gridDim.x >> 1), longer(n_longer), shorter(n_shorter)
    {
        rest = longer % pairs;
        // (a tile takes some three blocks beside its terms)
        const int each = rest == 0 ? 0 : (long_blocks + 3 + (short_blocks + 3) / 2) / (short_blocks + 3);
        ahead = (int)min((int64_t)shorter, (int64_t)(pairs - rest) * each);
    }
    // The n-th tile, of the longer product or the other; false after the last.
    __device__ __forceinline__ bool get(int n, bool &of_longer, int &i) const
    {
        const int first = longer > pair ? (longer - pair - 1) / pairs + 1 : 0;
        of_longer = n < first;
        if (of_longer) {
            i = pair + n * pairs;
            return true;
        }
        n -= first;
        const int own = pair - rest, many = pairs - rest, second = own >= 0 && ahead > own ? (ahead - own - 1) / many + 1 : 0;
        i = n < second ? own + n * many : ahead + pair + (n - second) * pairs;
        return i < shorter;
    }
};

__device__ __forceinline__ void add_box(const CUtensorMap *map, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
                 "r"(src), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

// Maximum and sum of exponentials below it: those of two sets of words.
__device__ __forceinline__ void join(float2 &a, float2 b)
{
    const float top = fmaxf(a.x, b.x);
    a = make_float2(top, a.y * exp2_fast((a.x - top) * kLog2e) + b.y * exp2_fast((b.x - top) * kLog2e));
}

// Logits: A is x (or packed), B w.  Products: of G (by its rows and by its columns) with w, and with x (or packed).
// 8,192 x 1,024 x 65,536, bf16: all logits 640 us (1.72 PFLOP/s, tensor cores active 71 % of the cycles); of 9,728 words G
// 133 us (55 %: a tile's stores, 128 KB a CTA, and what leads up to them take longer than its products), the products 411
// (1.59 PFLOP/s, 76 %, at the clock that power leaves).
template <class T, int kForm>
__global__ __cluster_dims__(2, 1, 1) __launch_bounds__(threads_of(kForm), 1) void head_kernel(
    const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap packed_map,
    const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap g_map,
    const __grid_constant__ CUtensorMap across_map, const __grid_constant__ CUtensorMap out_map,
    const __grid_constant__ CUtensorMap dw_map, const Params p)
{
    constexpr bool kLogits = of_logits(kForm);
    constexpr int kTeams = teams_of(kForm), kSlabs = slabs_of(kForm), kStages = stages_of(kForm);
    extern __shared__ uint8_t raw[];
    const uint32_t base = (smem_addr(raw) + 1023) & ~1023u;
    const uint32_t slabs = base + kStages * 2 * kHalf;
    const uint32_t bars = slabs + kTeams * kSlabs * kSlab;
    // barriers: full[stage], empty[stage], acc_full[2], acc_empty[2]
    const uint32_t full = bars, empty = bars + 8 * kStages, acc_full = bars + 16 * kStages, acc_empty = acc_full + 16;
    uint8_t *tail = raw + (bars + 16 * kStages + 32 - smem_addr(raw));
    volatile int *dead = reinterpret_cast<volatile int *>(tail);
    uint32_t *tmem_at = reinterpret_cast<uint32_t *>(tail) + 1;
    float2 *of_teams = reinterpret_cast<float2 *>(tail + 16);  // [2][team][row] (forward)

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank();

    if (threadIdx.x == 0) {
        *dead = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(full + 8 * s, 1);
            bar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(acc_full + 8 * s, 1);
            bar_init(acc_empty + 8 * s, 8 * kTeams);  // the teams' warps of either CTA
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_at)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(tmem_at);
    next_may_start();
    after_previous();

    const int count = p.shared->count, counted = count > 0 ? count : 1;
    const int row_tiles = (int)up(counted, kTile), word_tiles = (int)up(p.words, kTile), d_tiles = (int)up(p.d, kTile);
    Work dx, dw;  // (of the logits forms the first is theirs)
    if (kLogits) {
        dx = {row_tiles, word_tiles, (int)up(p.d, kBlockK), (int)up(p.d, kBlockK), 1};
        dw = {0, 0, 0, 0, 0};
    } else {
        dx = {row_tiles, d_tiles, (int)up(p.words, kBlockK), kValues * (int)up(p.words, kBlockK), p.dx_splits};
        dw = {word_tiles, d_tiles, (int)up(counted, kBlockK), kValues * (int)up(counted, kBlockK), p.dw_splits};
    }
    const int dx_length = dx.k_blocks / dx.splits, dw_length = kLogits ? 0 : dw.k_blocks / dw.splits;
    const bool dx_longer = dx_length >= dw_length;
    const Turns turns(dx_longer ? dx.tiles() : dw.tiles(), dx_longer ? dw.tiles() : dx.tiles(), dx_longer ? dx_length : dw_length,
                      dx_longer ? dw_length : dx_length);
    auto tile = [&](int n, bool &words, Tile &t) {  // the pair's n-th
        bool longer;
        int i;
        if (!turns.get(n, longer, i))
            return false;
        words = !kLogits && longer != dx_longer;
        t = tile_of(words ? dw : dx, i);
        return true;
    };
    const CUtensorMap *rows_map = count == p.rows ? &x_map : &packed_map;

    if (warp == 0) {
        if (lane == 0) {
            int step = 0;
            bool ok = true;
            bool words;
            Tile t;
            for (int n = 0; ok && tile(n, words, t); ++n) {
                const Work &work = words ? dw : dx;
                const int am = t.m * kTile + rank * kRowsCta, bn = t.n * kTile + (int)rank * kRowsCta;
                const CUtensorMap *b_map = words ? rows_map : &w_map;
                for (int k = t.k0; k < t.k1; ++k, ++step) {
                    const int s = step % kStages;
                    if (!(ok = bar_wait(empty + 8 * s, (step / kStages & 1) ^ 1, dead)))
                        break;
                    if (rank == 0)
                        bar_expect(full + 8 * s, 4 * kHalf);
                    const uint32_t bar = in_cta(full + 8 * s, 0), a = base + s * 2 * kHalf, b = a + kHalf;
                    if (kLogits) {
                        load_box(a, rows_map, k * kBlockK, am, bar);
                        load_box(b, &w_map, k * kBlockK, bn, bar);
                        continue;
                    }
                    // (what rounding left goes first, and so into sums of its own but for one part)
                    const int second = k < work.k_once, term = (k - (second ? 0 : work.k_once)) * kBlockK;
                    if (words) {
                        load_box(a, &across_map, am, term, second, bar);
                        load_box(a + kHalf / 2, &across_map, am + 64, term, second, bar);
                    } else {
                        load_box(a, &g_map, term, am, second, bar);
                    }
                    load_box(b, b_map, bn, term, bar);
                    load_box(b + kHalf / 2, b_map, bn + 64, term, bar);
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            // 32-bit sums, operands bf16 or f16, 256 x 256, each along its terms or its rows
            const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            const uint32_t kind0 = 1u << 4 | type << 7 | type << 10 | (uint32_t)!kLogits << 16 | (kTile / 8) << 17 | (kTile / 16) << 24;
            int step = 0, done = 0;
            bool ok = true;
            bool words;
            Tile t;
            for (int n = 0; ok && tile(n, words, t); ++n) {
                const uint32_t kind = kind0 | (uint32_t)words << 15;
                const int a_step = words ? 128 : 2;
                for (int k0 = t.k0;;) {  // (a part may have no terms)
                    const int k1 = min(k0 + part_of(kForm), t.k1), set = done & 1;
                    if (!(ok = bar_wait(acc_empty + 8 * set, (done >> 1 & 1) ^ 1, dead)))
                        break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t acc = tmem + set * kTile;
                    for (int k = k0; k < k1; ++k, ++step) {
                        const int s = step % kStages;
                        if (!(ok = bar_wait(full + 8 * s, step / kStages & 1, dead)))
                            break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t at = base + s * 2 * kHalf;
                        const uint64_t a = words ? operand<true>(at) : operand<false>(at), b = operand<!kLogits>(at + kHalf);
#pragma unroll
                        for (int q = 0; q < kBlockK / 16; ++q)  // 16 terms: 32 bytes on, or two groups of eight terms
                            multiply(acc, a + q * a_step, b + q * (kLogits ? 2 : 128), kind, k > k0 || q > 0);
                        commit(empty + 8 * s);
                    }
                    if (!ok)
                        break;
                    commit(acc_full + 8 * set);
                    ++done;
                    if ((k0 = k1) >= t.k1)
                        break;
                }
            }
        }
    } else {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const int team = (warp - 2) >> 2;
        const bool first = (threadIdx.x - 64) % 128 == 0;  // issues its team's stores
        const uint32_t slab0 = slabs + team * kSlabs * kSlab;
        const float back = kForm == kProducts && kScaled<T> ? 1.0f / p.shared->scale : 1.0f;
        constexpr int kCols = kTile / kTeams, kQ = kCols / 32;  // of a team's (logits)
        int done = 0, turn = 0;
        bool ok = true;
        auto release = [&](int set) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0)
                bar_arrive_cluster(in_cta(acc_empty + 8 * set, 0));
        };
        bool words;
        Tile t;
        for (int n = 0; tile(n, words, t); ++n) {
            const int m0 = t.m * kTile + rank * kRowsCta, at = m0 + row;
            const bool here = at < count;
            if constexpr (kLogits) {
                Slope slope{0.0f, 0.0f, 0.0f, -1};
                if (kForm == kSlopes && here)
                    slope = p.slopes[at];
                if (kForm == kStats && here)
                    slope.token = p.tokens[at];
                // the logits of this team's words, from their parts
                float l[kQ][32];
                auto part = [&] {  // where the next is
                    const int set = done & 1;
                    ok = __all_sync(~0u, ok && bar_wait(acc_full + 8 * set, done >> 1 & 1, dead));
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    return tmem + set * kTile + ((uint32_t)(quarter * 32) << 16) + team * kCols;
                };
                uint32_t acc = part();
#pragma unroll
                for (int q = 0; q < kQ; ++q)
                    load_acc(acc + q * 32, l[q]);
                wait_acc();
                release(done++ & 1);  // (the next products may take them)
#pragma unroll 1
                for (int k = t.k0 + part_of(kForm); k < t.k1; k += part_of(kForm)) {
                    acc = part();
#pragma unroll
                    for (int q = 0; q < 2 * kQ; ++q) {
                        float v[16];
                        load_acc(acc + q * 16, v);
                        wait_acc();
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            l[q >> 1][(q & 1) * 16 + e] += v[e];
                    }
                    release(done++ & 1);
                }
                // (past a wait that ran out all that follows is NaN, so that no wrong result passes for a right one)
                if (!ok) {
#pragma unroll
                    for (int q = 0; q < kQ; ++q)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            l[q][e] = __int_as_float(0x7fffffff);
                }
                const int word0 = t.n * kTile + team * kCols;
                if constexpr (kForm == kStats) {
                    float m = kLowest;
                    float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
                    for (int q = 0; q < kQ; ++q) {
                        const int word = word0 + q * 32;
                        if (slope.token >= word && slope.token < word + 32) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (slope.token == word + e)
                                    p.wanted[at] = l[q][e];
                        }
                        if (word + 32 > p.words) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                l[q][e] = word + e < p.words ? l[q][e] : no_value();
                        }
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            m = fmaxf(m, l[q][e]);
                    }
                    const float2 low = make_float2(-m, -m), c2 = make_float2(kLog2e, kLog2e);
#pragma unroll
                    for (int q = 0; q < kQ; ++q)
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const float2 u = mul2(add2(make_float2(l[q][e], l[q][e + 1]), low), c2);
                            sum = add2(sum, make_float2(exp2_fast(u.x), exp2_fast(u.y)));
                        }
                    // (the buffer of the tile before last: all have read it before they came to the last's barrier)
                    float2 *buffer = of_teams + (turn++ & 1) * kTeams * kRowsCta;
                    buffer[team * kRowsCta + row] = make_float2(m, sum.x + sum.y);
                    __syncwarp();
                    asm volatile("bar.sync %0, %1;" ::"n"(kTeams + 1), "n"(kTeams * 128) : "memory");
                    if (team == (turn & (kTeams - 1)) && here) {
                        float2 all = buffer[row];
#pragma unroll
                        for (int k = 1; k < kTeams; ++k)
                            join(all, buffer[k * kRowsCta + row]);
                        p.parts[(int64_t)t.n * p.rows + at] = all;
                    }
                } else {
                    // (shares as multiples of 2^-24: the fast exponential has nothing below 2^-126, of which sums over many
                    // rows would not be so small; the exponent's rounding is 2^-20 of the share then)
                    constexpr float kShift = 24.0f, kSmall = 1.0f / (1 << 24);
                    const float2 low = make_float2(-slope.m, -slope.m), c2 = make_float2(kLog2e, kLog2e),
                                 zc = make_float2(kShift - slope.z * kLog2e, kShift - slope.z * kLog2e),
                                 up = make_float2(-slope.up * kSmall, -slope.up * kSmall);
                    const int hit = slope.token - p.first - word0;  // of this team's words
                    // the token's own: of a share near one the others are what is left, which the shifted exponent's rounding
                    // would drown
                    float own = 0.0f;
                    if (hit >= 0 && hit < kCols) {
#pragma unroll
                        for (int q = 0; q < kQ; ++q)
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                own = hit == q * 32 + e ? l[q][e] : own;
                        if (p.wanted && ok)
                            own = p.wanted[at];
                        own = slope.up * one_less_exp((own - slope.m) - slope.z);
                    }
#pragma unroll
                    for (int q = 0; q < kQ; ++q) {
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            const float2 u = fma2(add2(make_float2(l[q][e], l[q][e + 1]), low), c2, zc);
                            const float2 g = mul2(make_float2(exp2_fast(u.x), exp2_fast(u.y)), up);
                            l[q][e] = g.x;
                            l[q][e + 1] = g.y;
                        }
                        if (hit >= q * 32 && hit < q * 32 + 32) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                l[q][e] = hit == q * 32 + e ? own : l[q][e];
                        }
                        // (rows past the last: x is 0 there, and 0 times what w holds may be NaN)
                        if (m0 + quarter * 32 + 32 > count) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                l[q][e] = here ? l[q][e] : 0.0f;
                        }
                        if (first)
                            stores_left<0>();
                        team_sync(team);
                        put32_in_two<T>(slab0, row, l[q]);
                        fence_async();
                        team_sync(team);
                        const int word = word0 + q * 32;
                        if (first && word < p.words && m0 < p.rows) {
                            store_box(&out_map, slab0, word, m0, 0);
                            store_box(&out_map, slab0 + kHalfSlab, word, m0, 1);
                        }
                        if (first)
                            stores_close();
                    }
                }
            } else {
                // this team's columns, summed over the parts of their terms
                float v[kQ][32];
                auto part = [&] {  // where the next is
                    const int set = done & 1;
                    ok = __all_sync(~0u, ok && bar_wait(acc_full + 8 * set, done >> 1 & 1, dead));
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    return tmem + set * kTile + ((uint32_t)(quarter * 32) << 16) + team * kCols;
                };
                uint32_t acc = part();
#pragma unroll
                for (int q = 0; q < kQ; ++q)
                    load_acc(acc + q * 32, v[q]);
                wait_acc();
                release(done++ & 1);  // (the next products may take them)
#pragma unroll 1
                for (int k = t.k0 + part_of(kForm); k < t.k1; k += part_of(kForm)) {
                    acc = part();
#pragma unroll
                    for (int q = 0; q < 2 * kQ; ++q) {
                        float u[16];
                        load_acc(acc + q * 16, u);
                        wait_acc();
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            v[q >> 1][(q & 1) * 16 + e] += u[e];
                    }
                    release(done++ & 1);
                }
                if (!ok || t.k0 >= t.k1) {  // (a part may have no terms)
                    const float other = ok ? 0.0f : __int_as_float(0x7fffffff);
#pragma unroll
                    for (int q = 0; q < kQ; ++q)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            v[q][e] = other;
                }
                // 16-bit results go 64 columns at a time, sums in 32 bits 32
                const bool parts = !words || p.dw_splits > 1;
                const CUtensorMap *out = words ? &dw_map : &out_map;
#pragma unroll
                for (int q = 0; q < kQ; ++q) {
                    const bool half = q & 1;
                    if (parts || !half) {
                        if (first)
                            stores_left<0>();
                        team_sync(team);
                    }
                    if (parts) {
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            put16(slab0, row, c, __float_as_uint(v[q][4 * c]), __float_as_uint(v[q][4 * c + 1]),
                                  __float_as_uint(v[q][4 * c + 2]), __float_as_uint(v[q][4 * c + 3]));
                    } else {
                        if (kScaled<T>) {
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                v[q][e] *= back;
                        }
                        put32<T>(slab0, row, half, v[q]);
                    }
                    if (!parts && !half)
                        continue;
                    fence_async();
                    team_sync(team);
                    const int c = t.n * kTile + team * kCols + (parts ? q : q & ~1) * 32;
                    if (first && c < p.d && m0 < (words ? p.words : p.rows)) {
                        if (!words && p.more)
                            add_box(out, slab0, c, m0, t.split);
                        else
                            store_box(out, slab0, c, m0, t.split);
                    }
                    if (first)
                        stores_close();
                }
            }
        }
        if (first)
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    __syncthreads();
    if (*dead)  // copies and products may still be under way
        linger();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols));
}

// ------------------------------------------------------------ few rows

// (8 x 1,024 x 65,536 31 us, on the tensor cores' tiles 43; 8 x 256 x 4,096 7.8 and 12.7)
constexpr int kFewRows = 8;
constexpr int kFewThreads = 128;
constexpr int kFewWords = 16 * (kFewThreads / 32);  // of a block

// c += a product of 16 words, 16 terms and eight rows, which is added in 32 bits: into its accumulator the instruction would
// truncate (of 2,048 terms, logits of 12 were off by 7e-6).
template <class T>
__device__ __forceinline__ void multiply_few(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    float p[4];
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(p[0]), "=f"(p[1]), "=f"(p[2]), "=f"(p[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(p[0]), "=f"(p[1]), "=f"(p[2]), "=f"(p[3])
            : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c[i] += p[i];
}

// The logits of 16 words, w0 and w1 a lane's, and up to eight rows of x, xr a lane's: a lane has words g and g + 8 of rows 2 t,
// 2 t + 1, t the lane's number among four (any order of the terms will do, as long as it is both's: a lane's 16 bytes are
// eight terms of one word, and of x the same eight of one row).  By whole warps: lanes whose terms are past the last go along
// with zeros.
template <class T, int kAhead>
__device__ __forceinline__ void few_logits(float (&c)[4], const T *w0, const T *w1, const T *xr, int64_t D, int t)
{
    float sums[2][4] = {};
#pragma unroll 1
    for (int64_t k0 = 0; k0 < D; k0 += 32 * kAhead) {
        uint4 a[kAhead], b[kAhead], v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t k = k0 + 32 * u + t * 8;
            a[u] = b[u] = v[u] = make_uint4(0, 0, 0, 0);
            if (k < D) {
                a[u] = __ldg(reinterpret_cast<const uint4 *>(w0 + k));
                b[u] = __ldg(reinterpret_cast<const uint4 *>(w1 + k));
                v[u] = __ldg(reinterpret_cast<const uint4 *>(xr + k));
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            multiply_few<T>(sums[0], a[u].x, b[u].x, a[u].y, b[u].y, v[u].x, v[u].y);
            multiply_few<T>(sums[1], a[u].z, b[u].z, a[u].w, b[u].w, v[u].z, v[u].w);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c[i] = sums[0][i] + sums[1][i];
}

// A warp takes 16 words against up to eight rows of x, which stay in L1: the table's bytes stream past once, straight
// into the operands of products of a warp.  Bound by the table's bytes: 4 x 1,024 x 65,536 27 us with what follows, 5.0
// TB/s (with half as many reads under way 29).
template <class T>
__global__ __launch_bounds__(kFewThreads, 7) void head_few_kernel(int rows, int64_t D, int64_t V, const T *x, int64_t xs, const T *w,
                                                               const void *tokens, int token_bytes, float2 *parts, float *wanted)
{
    constexpr int kWarps = kFewThreads / 32;
    __shared__ float2 of_warps[kWarps][kFewRows];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    next_may_start();
    const int64_t j0 = ((int64_t)blockIdx.x * kWarps + warp) * 16;
    const T *w0 = w + min(j0 + g, V - 1) * D, *w1 = w + min(j0 + g + 8, V - 1) * D, *xr = x + min(g, rows - 1) * xs;
    float c[4];
    few_logits<T, 4>(c, w0, w1, xr, D, t);
    // a lane has words j0 + g, j0 + g + 8 of rows 2 t, 2 t + 1
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 2 * t + i;
        const int64_t token = r < rows ? token_of(tokens, token_bytes, r) : -1;
        const float l0 = j0 + g < V ? c[i] : no_value(), l1 = j0 + g + 8 < V ? c[2 + i] : no_value();
        if (token >= 0 && token < V && (token == j0 + g || token == j0 + g + 8))
            wanted[r] = token == j0 + g ? l0 : l1;
        float m = fmaxf(fmaxf(l0, l1), kLowest);
#pragma unroll
        for (int o = 4; o < 32; o *= 2)
            m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
        float sum = exp2_fast((l0 - m) * kLog2e) + exp2_fast((l1 - m) * kLog2e);
#pragma unroll
        for (int o = 4; o < 32; o *= 2)
            sum += __shfl_xor_sync(~0u, sum, o);
        if (g == 0)
            of_warps[warp][r] = make_float2(m, sum);
    }
    __syncthreads();
    if (threadIdx.x < rows) {
        float2 q = of_warps[0][threadIdx.x];
        for (int k = 1; k < kWarps; ++k) {
            const float2 o = of_warps[k][threadIdx.x];
            const float top = fmaxf(q.x, o.x);
            q = make_float2(top, q.y * exp2_fast((q.x - top) * kLog2e) + o.y * exp2_fast((o.x - top) * kLog2e));
        }
        parts[(int64_t)threadIdx.x * gridDim.x + blockIdx.x] = q;
    }
}

// Backward, a warp a row: the logit of its token as `head_few_kernel` has summed it, so that of a row whose token is the peak
// l - m is 0.  (Of the tiles' sums it would be some 2^-21 of l, which of a confident row is more than what is left of one.)
template <class T>
__global__ __launch_bounds__(32, 1) void head_few_wanted_kernel(int rows, int64_t D, int64_t V, const T *x, int64_t xs, const T *w,
                                                             const void *tokens, int token_bytes, float *wanted)
{
    const int lane = threadIdx.x, t = lane & 3, r = blockIdx.x;
    next_may_start();
    const int64_t each = lane < rows ? token_of(tokens, token_bytes, lane) : -1, token = __shfl_sync(~0u, each, r);
    const int i = __popc(__ballot_sync(~0u, each >= 0 && each < V) & ((1u << r) - 1));  // of the packed rows
    float c[4] = {};
    if (token >= 0 && token < V) {
        const T *of_token = w + token * D;
        few_logits<T, 16>(c, of_token, of_token, x + min(lane >> 2, rows - 1) * xs, D, t);
    }
    after_previous();
    if (token >= 0 && token < V && lane == r >> 1)
        wanted[i] = c[r & 1];
}

// ------------------------------------------------------------ joining

constexpr int kJoinThreads = 512;

__device__ __forceinline__ void leave(int64_t r, bool has, float2 q, const float *wanted, float *logp, float *peak, float *logz)
{
    const float z = q.y != 0.0f ? logf(q.y) : no_value();  // (NaN counts)
    logp[r] = !has ? 0.0f : z == no_value() ? z : (*wanted - q.x) - z;
    if (peak)
        peak[r] = !has ? 0.0f : z == no_value() || (z != z && q.x != INFINITY) ? z : q.x;  // (NaN has not been compared)
    if (logz)
        logz[r] = has ? z : 0.0f;
}

// A row's maximum and sum from those of n parts, and what follows; lanes are rows.
__global__ __launch_bounds__(kJoinThreads) void head_join_kernel(int rows, const Shared *shared, const int *order, int n,
                                                                 const float2 *parts, const float *wanted, float *logp, float *peak,
                                                                 float *logz)
{
    constexpr int kWarps = kJoinThreads / 32, kAhead = 8;
    __shared__ float2 of_warps[kWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    next_may_start();
    after_previous();
    const int count = shared->count;
    float2 q = make_float2(kLowest, 0.0f);
    if (i < count) {
        for (int k = warp; k < n; k += kWarps * kAhead) {
            float2 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                v[u] = parts[(int64_t)min(k + u * kWarps, n - 1) * rows + i];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (k + u * kWarps < n)
                    join(q, v[u]);
        }
    }
    of_warps[warp][lane] = q;
    __syncthreads();
    if (warp > 0 || i >= count)
        return;
    for (int k = 1; k < kWarps; ++k)
        join(q, of_warps[k][lane]);
    leave(order[i], true, q, wanted + i, logp, peak, logz);
}

// The same of few rows, a block each, threads are parts.
__global__ __launch_bounds__(kJoinThreads) void head_join_few_kernel(int64_t V, const void *given, int token_bytes, int n,
                                                                     const float2 *parts, const float *wanted, float *logp,
                                                                     float *peak, float *logz)
{
    constexpr int kWarps = kJoinThreads / 32;
    __shared__ float2 of_warps[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = blockIdx.x;
    next_may_start();
    after_previous();
    float2 q = make_float2(kLowest, 0.0f);
#pragma unroll 4
    for (int k = threadIdx.x; k < n; k += kJoinThreads)
        join(q, parts[(int64_t)r * n + k]);
#pragma unroll
    for (int o = 16; o; o >>= 1)
        join(q, make_float2(__shfl_xor_sync(~0u, q.x, o), __shfl_xor_sync(~0u, q.y, o)));
    if (lane == 0)
        of_warps[warp] = q;
    __syncthreads();
    if (threadIdx.x > 0)
        return;
    for (int k = 1; k < kWarps; ++k)
        join(q, of_warps[k]);
    const int64_t t = token_of(given, token_bytes, r);
    leave(r, t >= 0 && t < V, q, wanted + r, logp, peak, logz);
}

// dx from its sums, parts in order, brought back from the scale; zeros in rows without a token.
template <class T>
__global__ __launch_bounds__(256) void head_dx_kernel(int rows, int64_t D, int splits, const float *sums, const int *place,
                                                      const Shared *shared, T *dx, int64_t dxs)
{
    next_may_start();
    after_previous();
    const float back = 1.0f / shared->scale;
    const int64_t per = D / 4, n = rows * per, all = rows * D / 4;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n; k += (int64_t)gridDim.x * 256) {
        const int64_t r = k / per, c = k % per;
        const int i = place[r];
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (i >= 0) {
            const float4 *from = reinterpret_cast<const float4 *>(sums) + i * per + c;
            v = from[0];
            for (int s = 1; s < splits; ++s) {
                const float4 q = from[s * all];
                v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
            }
            v.x *= back, v.y *= back, v.z *= back, v.w *= back;
        }
        *reinterpret_cast<uint2 *>(dx + r * dxs + c * 4) = make_uint2(pack2<T>(v.x, v.y), pack2<T>(v.z, v.w));
    }
}

// dw of a piece from its parts, in order.
template <class T>
__global__ __launch_bounds__(256) void head_dw_kernel(int64_t n, int splits, const float *parts, const Shared *shared, T *dw)
{
    next_may_start();
    after_previous();
    const float back = 1.0f / shared->scale;
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < n / 4; k += (int64_t)gridDim.x * 256) {
        float4 v = reinterpret_cast<const float4 *>(parts)[k];
        for (int s = 1; s < splits; ++s) {
            const float4 q = reinterpret_cast<const float4 *>(parts)[k + s * (n / 4)];
            v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
        }
        reinterpret_cast<uint2 *>(dw)[k] = make_uint2(pack2<T>(v.x * back, v.y * back), pack2<T>(v.z * back, v.w * back));
    }
}

// ------------------------------------------------------------ host

// Into how many parts the terms of the two products of a piece are dealt, of `rows` rows and `words` words: those that end
// soonest, and when, in us.  A block of 64 terms takes a pair 0.27 us, a tile 0.8
// us beside them, and sums in parts a pass that adds them up (of dw, a launch too).
double deal(int64_t rows, int64_t words, int64_t D, int &dx_splits, int &dw_splits)
{
    const int64_t across = up(D, kTile), dx_tiles = up(rows, kTile) * across, dw_tiles = up(words, kTile) * across;
    const int64_t dx_blocks = kValues * up(words, kBlockK), dw_blocks = kValues * up(rows, kBlockK);
    double least = 0.0;
    constexpr int kTried[] = {1, 2, 3, 4, 6, 8, 12, 16};
    for (int a : kTried)
        for (int b : kTried) {
            if (a > dx_blocks || b > dw_blocks)
                break;
            const double l1 = 0.27 * up(dx_blocks, a) + 0.8, l2 = 0.27 * up(dw_blocks, b) + 0.8;
            // the longer's tiles go round, the other's level what that leaves
            const bool first = l1 >= l2;
            const int64_t n1 = first ? dx_tiles * a : dw_tiles * b, n2 = first ? dw_tiles * b : dx_tiles * a, rest = n1 % kPairs;
            const double more = first ? l1 : l2, less = first ? l2 : l1;
            const int64_t each = rest ? (int64_t)(more / less + 0.5) : 0, ahead = n2 < (kPairs - rest) * each ? n2 : (kPairs - rest) * each;
            const int64_t round = up(n2 - ahead, kPairs);
            const double high = (n1 / kPairs + (rest > 0)) * more + round * less,
                         low = n1 / kPairs * more + (up(ahead, kPairs - rest) + round) * less;
            double us = high > low ? high : low;
            us += (double)rows * D * 4 * a / 5e6 + (b > 1 ? 3.0 + (double)words * D * 8 * b / 5e6 : 0.0);
            if (least == 0.0 || us < least) {
                least = us;
                dx_splits = a;
                dw_splits = b;
            }
        }
    return least;
}

// Values of G at once: 470 MB as two.  Backward, with 134, 336, 470 and 671 MB: 8,192 x 256 x 32,768 770, 724, 665 and
// 654 us, 16,384 x 512 x 32,768 2.32, 2.01, 1.97 and 1.93 ms; 8,192 x 1,024 x 65,536 3.95, 3.86, 3.82 and 3.71.
constexpr int64_t kPieceValues = int64_t(7) << 24;

// Words at once: the number that ends soonest, of those that leave G in its room.  (With room for 336 MB, 2,999 x 520 x
// 50,021: 25,856 words at a time 533 us by these estimates, the most that there was room for 559.)  A tile of logits takes a pair its
// products, or some 5 us to its slopes and stores.
int64_t piece_of(int64_t rows, int64_t D, int64_t V)
{
    const int64_t most = kPieceValues / rows / kTile > 4 ? kPieceValues / rows / kTile : 4, all = up(V, kTile);
    if (all <= most)
        return up(V, 64) * 64;
    const double logits = 0.27 * up(D, kBlockK) > 5.0 ? 0.27 * up(D, kBlockK) : 5.0;
    auto takes = [&](int64_t tiles) {
        int a, b;
        return deal(rows, tiles * kTile, D, a, b) + logits * up(up(rows, kTile) * tiles, kPairs) + 6.0;
    };
    int64_t best = most;
    double least = 0.0;
    for (int64_t k = most; k > most / 2 && most - k < 64; --k) {
        const int64_t pieces = up(all, k);
        const double us = (pieces - 1) * takes(k) + takes(all - (pieces - 1) * k);
        if (least == 0.0 || us < least) {
            least = us;
            best = k;
        }
    }
    return best * kTile;
}

struct Layout {
    int64_t shared, order, place, tokens, slopes, packed, parts, wanted, g, dx, dw, bytes;
    int64_t piece;  // words at once
    int dx_splits, dw_splits;
};

Layout make_layout(int64_t rows, int64_t D, int64_t V, bool grad)
{
    Layout l{};
    auto take = [&](int64_t bytes) {
        const int64_t at = l.bytes;
        l.bytes += up(bytes, 256) * 256;
        return at;
    };
    if (!grad && rows <= kFewRows) {
        l.parts = take(up(V, kFewWords) * rows * 8);
        l.wanted = take(rows * 4);
        return l;
    }
    l.shared = take(sizeof(Shared));
    l.order = take(rows * 4);
    l.place = take(rows * 4);
    l.packed = take(rows * D * 2);
    if (!grad) {
        l.tokens = take(rows * 4);
        l.parts = take(up(V, kTile) * rows * 8);
        l.wanted = take(rows * 4);
        return l;
    }
    l.slopes = take(rows * (int64_t)sizeof(Slope));
    l.wanted = take(rows <= kFewRows ? rows * 4 : 0);
    l.piece = piece_of(rows, D, V);
    const int64_t words = l.piece < V ? l.piece : V;
    deal(rows, words, D, l.dx_splits, l.dw_splits);
    l.g = take(kValues * rows * l.piece * 2);
    l.dx = take(l.dx_splits * rows * D * 4);
    l.dw = take(l.dw_splits > 1 ? l.dw_splits * words * D * 4 : 0);
    return l;
}

// The same, remembered by its sizes: a call asks for it three times, and pieces are chosen in some 100 us.
const Layout &layout_of(int64_t rows, int64_t D, int64_t V, bool grad)
{
    struct Known {
        int64_t rows, D, V;
        Layout layout;
    };
    static thread_local Known known[2] = {{-1, 0, 0, {}}, {-1, 0, 0, {}}};
    Known &k = known[grad];
    if (k.rows != rows || k.D != D || k.V != V)
        k = {rows, D, V, make_layout(rows, D, V, grad)};
    return k.layout;
}

template <class T, int kForm>
cudaError_t go(const CUtensorMap &x, const CUtensorMap &packed, const CUtensorMap &w, const CUtensorMap &g, const CUtensorMap &across,
               const CUtensorMap &out, const CUtensorMap &dw, const Params &p, int64_t tiles, cudaStream_t st)
{
    const auto kernel = head_kernel<T, kForm>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(kForm));
    if (e != cudaSuccess)
        return e;
    return launch_chained(kernel, 2 * (unsigned)(tiles < kPairs ? tiles : kPairs), threads_of(kForm), smem_of(kForm), st, true, x, packed, w, g,
                          across, out, dw, p);
}

unsigned blocks_for(int64_t n)
{
    const int64_t b = up(n, 256);
    return (unsigned)(b < 1 ? 1 : b < 152 * 8 ? b : 152 * 8);
}

// The rows that have a token, packed, and what goes with them.
template <bool kGrad, bool kScale>
cudaError_t prepare_rows(const HeadArgs &a, char *base, const Layout &l, float *logp, float *peak, float *logz, const float *dlogp,
                         cudaStream_t st)
{
    const int rows = (int)a.rows;
    const int64_t xs = rows > 1 ? a.x_stride : a.D;
    Shared *shared = reinterpret_cast<Shared *>(base + l.shared);
    int *order = reinterpret_cast<int *>(base + l.order), *place = reinterpret_cast<int *>(base + l.place),
        *tokens = reinterpret_cast<int *>(base + l.tokens);
    Slope *slopes = reinterpret_cast<Slope *>(base + l.slopes);
    const uint4 *x = (const uint4 *)a.x;
    uint4 *packed = reinterpret_cast<uint4 *>(base + l.packed);
    if (rows <= kOnceRows) {
        head_once_kernel<kGrad, kScale><<<(unsigned)up(rows, kOnceEach), kOnceThreads, 0, st>>>(
            rows, a.V, a.tokens, a.token_bytes, order, place, tokens, shared, logp, peak, logz, dlogp, slopes, a.D, x, xs, packed);
        return cudaGetLastError();
    }
    head_rows_kernel<kGrad, kScale><<<1, kRowsThreads, 0, st>>>(rows, a.V, a.tokens, a.token_bytes, order, place, tokens, shared, logp,
                                                                peak, logz, dlogp, slopes);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess)
        return e;
    return launch_chained(head_pack_kernel, blocks_for(a.rows * a.D / 8), 256, 0, st, true, rows, a.D, x, xs, (const int *)order,
                          (const Shared *)shared, packed);
}

}  // namespace

int64_t head_work_bytes(int64_t rows, int64_t D, int64_t V, bool grad) { return rows ? layout_of(rows, D, V, grad).bytes : 0; }

cudaError_t launch_head(const HeadArgs &a, float *logp, float *peak, float *logz, void *work, cudaStream_t st)
{
    if (!map_encoder())
        return cudaErrorNotSupported;
    const Layout &l = layout_of(a.rows, a.D, a.V, false);
    char *base = (char *)work;
    float2 *parts = reinterpret_cast<float2 *>(base + l.parts);
    float *wanted = reinterpret_cast<float *>(base + l.wanted);
    const int rows = (int)a.rows;
    auto run = [&](auto v) {
        using T = decltype(v);
        cudaError_t e;
        if (rows <= kFewRows) {
            const int blocks = (int)up(a.V, kFewWords);
            head_few_kernel<T><<<blocks, kFewThreads, 0, st>>>(rows, a.D, a.V, (const T *)a.x, rows > 1 ? a.x_stride : a.D,
                                                               (const T *)a.w, a.tokens, a.token_bytes, parts, wanted);
            e = cudaGetLastError();
            if (e != cudaSuccess)
                return e;
            return launch_chained(head_join_few_kernel, rows, kJoinThreads, 0, st, true, a.V, a.tokens, a.token_bytes, blocks, parts,
                                  wanted, logp, peak, logz);
        }
        Shared *shared = reinterpret_cast<Shared *>(base + l.shared);
        int *order = reinterpret_cast<int *>(base + l.order), *tokens = reinterpret_cast<int *>(base + l.tokens);
        e = prepare_rows<false, false>(a, base, l, logp, peak, logz, nullptr, st);
        if (e != cudaSuccess)
            return e;
        CUtensorMap x, packed, w;
        if (!operand_map(&x, a.dtype, a.x, rows, a.D, a.x_stride, kRowsCta) ||
            !operand_map(&packed, a.dtype, base + l.packed, rows, a.D, a.D, kRowsCta) ||
            !operand_map(&w, a.dtype, a.w, a.V, a.D, a.D, kRowsCta))
            return cudaErrorInvalidValue;
        Params p{};
        p.rows = rows;
        p.words = (int)a.V;
        p.d = (int)a.D;
        p.shared = shared;
        p.tokens = tokens;
        p.parts = parts;
        p.wanted = wanted;
        e = go<T, kStats>(x, packed, w, w, w, w, w, p, up(rows, kTile) * up(a.V, kTile), st);
        if (e != cudaSuccess)
            return e;
        return launch_chained(head_join_kernel, (unsigned)up(rows, 32), kJoinThreads, 0, st, true, rows, shared, order,
                              (int)up(a.V, kTile), parts, wanted, logp, peak, logz);
    };
    return a.dtype == AV_BF16 ? run(__nv_bfloat16()) : run(__half());
}

cudaError_t launch_head_grad(const HeadArgs &a, const float *dlogp, const float *peak, const float *logz, void *dx, int64_t dx_stride,
                             void *dw, void *work, cudaStream_t st)
{
    if (!map_encoder())
        return cudaErrorNotSupported;
    const Layout &l = layout_of(a.rows, a.D, a.V, true);
    char *base = (char *)work;
    const int rows = (int)a.rows;
    auto run = [&](auto v) {
        using T = decltype(v);
        Shared *shared = reinterpret_cast<Shared *>(base + l.shared);
        int *place = reinterpret_cast<int *>(base + l.place);
        cudaError_t e = prepare_rows<true, kScaled<T>>(a, base, l, nullptr, const_cast<float *>(peak), const_cast<float *>(logz), dlogp, st);
        if (e != cudaSuccess)
            return e;
        float *wanted = rows <= kFewRows ? reinterpret_cast<float *>(base + l.wanted) : nullptr;
        if (wanted)
            e = launch_chained(head_few_wanted_kernel<T>, rows, 32, 0, st, true, rows, a.D, a.V, (const T *)a.x,
                               rows > 1 ? a.x_stride : a.D, (const T *)a.w, a.tokens, a.token_bytes, wanted);
        if (e != cudaSuccess)
            return e;
        float *sums = reinterpret_cast<float *>(base + l.dx), *dw_parts = reinterpret_cast<float *>(base + l.dw);
        CUtensorMap x, packed, xt, packedt, dx_map;
        const int64_t dx_dims[3] = {a.D, rows, l.dx_splits}, dx_strides[2] = {a.D, rows * a.D};
        const int wide[3] = {32, kRowsCta, 1}, full[3] = {64, kRowsCta, 1}, across[3] = {64, 64, 1};
        if (!operand_map(&x, a.dtype, a.x, rows, a.D, a.x_stride, kRowsCta) ||
            !operand_map(&packed, a.dtype, base + l.packed, rows, a.D, a.D, kRowsCta) ||
            !operand_map(&xt, a.dtype, a.x, rows, a.D, a.x_stride, 64) ||
            !operand_map(&packedt, a.dtype, base + l.packed, rows, a.D, a.D, 64) ||
            !make_map(&dx_map, AV_F32, sums, 3, dx_dims, dx_strides, wide))
            return cudaErrorInvalidValue;
        for (int64_t j = 0; j < a.V; j += l.piece) {
            const int64_t words = a.V - j < l.piece ? a.V - j : l.piece;
            const T *w = (const T *)a.w + j * a.D;
            T *dwp = (T *)dw + j * a.D;
            const int64_t g_dims[3] = {words, rows, kValues}, g_strides[2] = {l.piece, l.piece * rows};
            CUtensorMap wk, wt, g_out, g, gt, dw_map;
            if (!operand_map(&wk, a.dtype, w, words, a.D, a.D, kRowsCta) || !operand_map(&wt, a.dtype, w, words, a.D, a.D, 64) ||
                !make_map(&g_out, a.dtype, base + l.g, 3, g_dims, g_strides, wide, CU_TENSOR_MAP_SWIZZLE_64B) ||
                !make_map(&g, a.dtype, base + l.g, 3, g_dims, g_strides, full) ||
                !make_map(&gt, a.dtype, base + l.g, 3, g_dims, g_strides, across))
                return cudaErrorInvalidValue;
            const int64_t dw_dims[3] = {a.D, words, l.dw_splits}, dw_strides[2] = {a.D, words * a.D};
            if (!(l.dw_splits > 1 ? make_map(&dw_map, AV_F32, dw_parts, 3, dw_dims, dw_strides, wide)
                                  : make_map(&dw_map, a.dtype, dwp, 3, dw_dims, dw_strides, full)))
                return cudaErrorInvalidValue;
            Params p{};
            p.rows = rows;
            p.words = (int)words;
            p.first = (int)j;
            p.d = (int)a.D;
            p.dx_splits = l.dx_splits;
            p.dw_splits = l.dw_splits;
            p.more = j > 0;
            p.shared = shared;
            p.slopes = reinterpret_cast<const Slope *>(base + l.slopes);
            p.wanted = wanted;
            e = go<T, kSlopes>(x, packed, wk, g, g, g_out, g_out, p, up(rows, kTile) * up(words, kTile), st);
            if (e != cudaSuccess)
                return e;
            e = go<T, kProducts>(xt, packedt, wt, g, gt, dx_map, dw_map, p,
                                 (up(rows, kTile) * p.dx_splits + up(words, kTile) * p.dw_splits) * up(a.D, kTile), st);
            if (e == cudaSuccess && l.dw_splits > 1)
                e = launch_chained(head_dw_kernel<T>, blocks_for(words * a.D / 4), 256, 0, st, true, words * a.D, l.dw_splits,
                                   (const float *)dw_parts, (const Shared *)shared, dwp);
            if (e != cudaSuccess)
                return e;
        }
        return launch_chained(head_dx_kernel<T>, blocks_for(rows * a.D / 4), 256, 0, st, true, rows, a.D, l.dx_splits,
                              (const float *)sums, (const int *)place, (const Shared *)shared, (T *)dx, rows > 1 ? dx_stride : a.D);
    };
    return a.dtype == AV_BF16 ? run(__nv_bfloat16()) : run(__half());
}

}  // namespace av
