// k_ffn.cu -- the gated feed-forward and its gradient.
//   forward   g = x wg^T, u = x wu^T, h = act(g) u
//   backward  dg = dh u act'(g), du = dh act(g); dx = dg wg + du wu; dwg = dg^T x, dwu = du^T x
//
// The products run on the tensor cores (tcgen05, accumulators in TMEM): one
// persistent kernel in four forms, a pair of CTAs on a tile of 256 rows x 256
// columns.  Per 64 terms a CTA fetches 128 rows of A and 128 of B (32 KB) for
// 512 cycles of products; alone, a CTA on 128 x 256 would fetch 48 KB in the
// same time, 96 bytes a cycle, more than an SM gets from L2.  In the forward
// form the pair's 256 columns are 128 of the gate and 128 of the same columns
// of the other projection, so one CTA's accumulators hold both factors of its
// outputs and h leaves rounded once, with no array in between.  The backward
// pass makes g and u again (4 M D H operations of 16) instead of keeping them:
// kept in 16 bits they would cost accuracy, in 32 bits 8 bytes a unit.  dg and du
// go to the last products as two values of 16 bits each, the rounded one and
// what it leaves, and the products take both: 24 M D H operations in all, but
// only the results are rounded.  (Rounded once in between, dx and dw were off by
// 1.41 times as much, as root mean square.)  float16 has not the range for them:
// they go times a power of two, which a bound on their largest gives
// (`ffn_peaks_kernel`), and the results are brought back before they are rounded.
//
// Warps: one issues copies (TMA), one products, four or eight take accumulators
// to memory while the next tile's products run (two sets of 256 TMEM columns).
// The gated forms take eight: with four the backward one spent more time on
// activations than on products (16,384 x 1,024 x 4,096: 204 us).
#include "async.cuh"
#include "policy.h"
#include "tensor_map.h"
#include "values.cuh"

namespace av {
namespace {

// ------------------------------------------------------------ activations

// act(g) and its slope.  exp and the divide are the fast ones: the exponential is
// good to 2 + 1.17 |g| units of 2^-23 (gelu: of the cubic), so the activation to
// 2^-21 relatively near 0 and 2^-16 where it all but vanishes at |g| = 88, less
// than a tenth of the outputs' rounding.
template <int kAct>
__device__ __forceinline__ void activate(float g, float &f, float &slope)
{
    // both are g times a sigmoid: of g, or of 2 sqrt(2/pi) (g + 0.044715 g^3)
    const float c = 1.5957691216057308f, in = kAct == AV_SILU ? g : c * (g + 0.044715f * g * g * g);
    const float s = __fdividef(1.0f, 1.0f + __expf(-in));
    f = g * s;
    const float din = kAct == AV_SILU ? 1.0f : c * (1.0f + 3.0f * 0.044715f * g * g);
    slope = s + f * (1.0f - s) * din;
}

constexpr int kValues = 2;  // that dg and du go as: [row][value][dg, du][H]

// What rounding to T leaves of v; nothing of infinity and NaN.
template <class T>
__device__ __forceinline__ float left_of(float v)
{
    const float r = to_f32(from_f32<T>(v));
    return fabsf(r) <= 3.402823466e38f ? v - r : 0.0f;
}

// ------------------------------------------------------------ float16's range

template <class T>
__device__ __forceinline__ void unpack8(const uint4 &v, float *f)
{
    const T *p = reinterpret_cast<const T *>(&v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        f[i] = to_f32(p[i]);
}

template <class T>
constexpr bool kScaled = std::is_same<T, __half>::value;
constexpr int kPeakThreads = 256;

// What bounds dg and du: the largest |dh|, and the largest sums of squares of a
// row of x and of w; each in 32 places, of which the largest counts.
using Peaks = const float4 *;
constexpr int kPeakBytes = 32 * 16;

// A power of two that brings dg and du below 2^15: |dg| <= |dh| |u| 1.13 and |du|
// <= |dh| |g|, projections are no larger than the product of their rows'
// lengths.  The bound is some ten times the largest value, so this is good to
// 2^-22 and, of the smallest, 2^-36 of the largest.  For whole warps.
__device__ __forceinline__ float scale_of(Peaks p)
{
    float4 v = p[threadIdx.x & 31];
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x = fmaxf(v.x, __shfl_xor_sync(~0u, v.x, o));
        v.y = fmaxf(v.y, __shfl_xor_sync(~0u, v.y, o));
        v.z = fmaxf(v.z, __shfl_xor_sync(~0u, v.z, o));
    }
    const float most = 1.16f * v.x * sqrtf(v.y) * sqrtf(v.z);
    if (!(most > 0.0f))
        return 1.0f;
    const int k = 15 - ((int)(__float_as_uint(most) >> 23) - 126);  // (most < 2^(exponent - 126))
    return __int_as_float((127 + min(max(k, -60), 60)) << 23);
}

// The peaks, of finite values; they are zeroed before.  A warp takes a row, of dh,
// x or w by the block's y; maxima do not depend on their order.  4,099 x 520 x
// 1,368 some 8 us, 65,536 x 256 x 512 21, both from memory.
template <class T>
__global__ __launch_bounds__(kPeakThreads) void ffn_peaks_kernel(int64_t rows, int64_t D, int64_t H, const T *x, int64_t xs,
                                                                 const T *w, const T *dh, int64_t dhs, float4 *peaks)
{
    constexpr int kWarps = kPeakThreads / 32;
    __shared__ float of_warps[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.y;
    const T *from = which == 0 ? dh : which == 1 ? x : w;
    const int64_t n = which == 0 ? H : D, count = which == 2 ? 2 * H : rows, stride = which == 0 ? dhs : which == 1 ? xs : D;
    float most = 0.0f;
    for (int64_t r = (int64_t)blockIdx.x * kWarps + warp; r < count; r += (int64_t)gridDim.x * kWarps) {
        const T *row = from + r * stride;
        float sum = 0.0f, top = 0.0f;
#pragma unroll 8
        for (int64_t k = lane * 8; k < n; k += 256) {
            float v[8];
            unpack8<T>(__ldg(reinterpret_cast<const uint4 *>(row + k)), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = fabsf(v[e]) <= 3.402823466e38f ? fabsf(v[e]) : 0.0f;
                sum = fmaf(a, a, sum);
                top = fmaxf(top, a);
            }
        }
        if (which != 0) {
#pragma unroll
            for (int o = 16; o; o >>= 1)
                sum += __shfl_xor_sync(~0u, sum, o);
        }
        most = fmaxf(most, which == 0 ? top : sum);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1)
        most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
    if (lane == 0)
        of_warps[warp] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 0; k < kWarps; ++k)
            most = fmaxf(most, of_warps[k]);
        atomicMax(reinterpret_cast<int *>(peaks + (blockIdx.x & 31)) + which, __float_as_int(most));  // (none is negative)
    }
}

// ------------------------------------------------------------ few rows

constexpr int kFewRows = 4;  // (eight: 18.6 us, 16: 28.8, by tensor cores 12.5, at 1,024 x 4,096)
constexpr int kFewThreads = 256;

// A warp per unit of H: its two rows of weights stream past, 16 bytes a lane,
// against R rows of x that stay in L1.  Bound by the weights' bytes: 4 x 1,024 x
// 4,096 8.2 us, 2.0 TB/s, of which some 3 are the launch.
template <class T, int kAct, int R, bool kGrad>
__global__ __launch_bounds__(kFewThreads) void ffn_few_kernel(int rows, int64_t D, int64_t H, const T *x, int64_t xs,
                                                               const T *w, T *h, int64_t hs, const T *dh, int64_t dhs,
                                                               T *dgu, Peaks peaks)
{
    const int lane = threadIdx.x & 31;
    const int64_t j = (int64_t)blockIdx.x * (kFewThreads / 32) + (threadIdx.x >> 5);
    if constexpr (kGrad)
        next_may_start();
    if (j >= H)
        return;
    const T *wg = w + j * D, *wu = w + (H + j) * D;
    const float scale = kGrad && kScaled<T> ? scale_of(peaks) : 1.0f;
    float g[R] = {}, u[R] = {};
#pragma unroll 2
    for (int64_t k = lane * 8; k < D; k += 256) {
        float a[8], b[8];
        unpack8<T>(__ldg(reinterpret_cast<const uint4 *>(wg + k)), a);
        unpack8<T>(__ldg(reinterpret_cast<const uint4 *>(wu + k)), b);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= rows)
                break;
            float v[8];
            unpack8<T>(__ldg(reinterpret_cast<const uint4 *>(x + r * xs + k)), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[r] += v[i] * a[i];
                u[r] += v[i] * b[i];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            g[r] += __shfl_xor_sync(~0u, g[r], o);
            u[r] += __shfl_xor_sync(~0u, u[r], o);
        }
        if (lane != r || r >= rows)
            continue;
        float f, slope;
        activate<kAct>(g[r], f, slope);
        if (!kGrad) {
            h[r * hs + j] = from_f32<T>(f * u[r]);
        } else {
            const float d = to_f32(dh[r * dhs + j]) * scale, dg = d * u[r] * slope, du = d * f;
            T *to = dgu + r * 2 * kValues * H + j;
            to[0] = from_f32<T>(dg);
            to[H] = from_f32<T>(du);
            to[2 * H] = from_f32<T>(left_of<T>(dg));
            to[3 * H] = from_f32<T>(left_of<T>(du));
        }
    }
}

// ------------------------------------------------------------ products

constexpr int kRowsCta = 128;  // accumulator rows of a CTA, and B rows it fetches
constexpr int kTile = 256;     // rows and columns of a pair's tile
constexpr int kBlockK = 64;    // terms a stage: 128 bytes, the swizzle's width
constexpr int kHalf = kRowsCta * kBlockK * 2;  // bytes of A or of B a CTA fetches per stage
constexpr int kSlab = kRowsCta * 128;  // staging of 128 rows x 128 bytes on the way out
constexpr int kHalfSlab = kSlab / 2;   // of 64 bytes
constexpr int kTmemCols = 512;

enum Form {
    kForward,  // h
    kProjGrad, // dg, du from dh and the projections made again
    kTimesW,   // dx = dgu w: B runs along its rows
    kTransposed // dw = dgu^T x: A and B run along their rows
};

// Fours of warps that take accumulators out; slabs of each; stages of A and B.
__host__ __device__ constexpr int teams_of(int form) { return form == kForward || form == kProjGrad ? 2 : 1; }
__host__ __device__ constexpr int slabs_of(int form) { return form == kForward ? 1 : 2; }
__host__ __device__ constexpr int stages_of(int form) { return form == kProjGrad ? 5 : 6; }
__host__ __device__ constexpr int threads_of(int form) { return 64 + 128 * teams_of(form); }
__host__ __device__ constexpr int smem_of(int form)
{
    return stages_of(form) * 2 * kHalf + teams_of(form) * slabs_of(form) * kSlab + 1024 + 256;
}

struct Params {
    int m, n;               // rows and columns of the result (forward forms: columns of H)
    int m_tiles, n_tiles;   // of a pair
    int k_blocks, splits;   // blocks of 64 terms in all, parts that they are dealt to
    int k_once;             // of them those of A's second value, which come first; B's come again for the first
    const void *dh;
    int64_t dhs;
    Peaks peaks;            // what dg and du are scaled by, of float16
};

__device__ __forceinline__ uint32_t cta_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// A box of a tensor map to this CTA's shared memory; the bytes are counted at
// a barrier of the pair's first CTA.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
                 "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
                 "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}

__device__ __forceinline__ void store_box(const CUtensorMap *map, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
                 "r"(src), "r"(x), "r"(y), "r"(z)
                 : "memory");
}

// Closes a group of stores, which may be empty: slabs are counted by groups.
__device__ __forceinline__ void stores_close() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void stores_left()
{
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}

// Shared-memory operand, 128-byte swizzle.  Along its terms (K-major): rows of
// 128 bytes, groups of eight rows 1024 bytes apart.  Along its rows
// (MN-major): boxes of 64 rows x 64 terms, a term's 64 rows in 128 bytes,
// groups of eight terms 1024 bytes apart, the next 64 rows 8192 bytes on.
template <bool kAlongRows>
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    const uint64_t lead = kAlongRows ? 8192 >> 4 : 1, group = 1024 >> 4;
    return (uint64_t)(addr >> 4 & 0x3fff) | lead << 16 | group << 32 | 1ull << 46 | 2ull << 61;
}

__device__ __forceinline__ void multiply(uint32_t acc, uint64_t a, uint64_t b, uint32_t kind, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(acc),
                 "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add)
                 : "memory");
}

// The barrier, in both CTAs, when all products issued so far are done.
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}

// 32 columns of this thread's accumulator row.
__device__ __forceinline__ void load_acc(uint32_t addr, float (&v)[32])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
                   "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
                   "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
                   "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
}

__device__ __forceinline__ void wait_acc() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

template <class T>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    T v[2] = {from_f32<T>(a), from_f32<T>(b)};
    return *reinterpret_cast<uint32_t *>(v);
}

// 16 bytes of a row into a staging slab, in the 128-byte swizzle; of 64-byte
// rows, in the 64-byte swizzle.
__device__ __forceinline__ void put16(uint32_t slab, int row, int chunk, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t at = slab + row * 128 + ((chunk ^ (row & 7)) << 4);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void put16_narrow(uint32_t slab, int row, int chunk, uint32_t a, uint32_t b, uint32_t c,
                                             uint32_t d)
{
    const uint32_t at = slab + row * 64 + ((chunk ^ (row >> 1 & 3)) << 4);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

template <class T>
__device__ __forceinline__ void put32(uint32_t slab, int row, int half, const float (&v)[32])
{
#pragma unroll
    for (int c = 0; c < 4; ++c)
        put16(slab, row, half * 4 + c, pack2<T>(v[8 * c], v[8 * c + 1]), pack2<T>(v[8 * c + 2], v[8 * c + 3]),
              pack2<T>(v[8 * c + 4], v[8 * c + 5]), pack2<T>(v[8 * c + 6], v[8 * c + 7]));
}

// As two values, to a half slab each.
template <class T>
__device__ __forceinline__ void put32_in_two(uint32_t slab, int row, const float (&v)[32])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float *q = v + 8 * c;
        put16_narrow(slab, row, c, pack2<T>(q[0], q[1]), pack2<T>(q[2], q[3]), pack2<T>(q[4], q[5]), pack2<T>(q[6], q[7]));
        put16_narrow(slab + kHalfSlab, row, c, pack2<T>(left_of<T>(q[0]), left_of<T>(q[1])),
                     pack2<T>(left_of<T>(q[2]), left_of<T>(q[3])), pack2<T>(left_of<T>(q[4]), left_of<T>(q[5])),
                     pack2<T>(left_of<T>(q[6]), left_of<T>(q[7])));
    }
}

__device__ __forceinline__ void team_sync(int team)
{
    __syncwarp();
    asm volatile("bar.sync %0, 128;" ::"r"(team + 1) : "memory");
}

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

struct Tile {
    int m, n, k0, k1, split;
};

// Tiles in bands of eight rows of tiles, down the band first: those in flight
// together share A and B in L2.
__device__ __forceinline__ Tile tile_of(const Params &p, int i)
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

// 16,384 x 1,024 x 4,096, bf16: h 156 us (1.76 PFLOP/s, tensor cores active 79 %
// of the cycles, at the clock that power leaves), dg and du 243 (49 %: dh's loads,
// the activations' gradients and the stores of two values), dx 319 and dw 310
// (96 %), of two values twice the products.
template <class T, int kForm, int kAct, bool kParts>
__global__ __cluster_dims__(2, 1, 1) __launch_bounds__(threads_of(kForm), 1) void ffn_kernel(
    const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
    const __grid_constant__ CUtensorMap out_map, const Params p)
{
    constexpr bool kARows = kForm == kTransposed, kBRows = kForm == kTimesW || kForm == kTransposed;
    constexpr bool kGated = kForm == kForward || kForm == kProjGrad;
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

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cta_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int tiles = p.m_tiles * p.n_tiles * p.splits;

    if (threadIdx.x == 0) {
        *dead = 0;
        for (int s = 0; s < kStages; ++s) {
            bar_init(full + 8 * s, 1);
            bar_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < 2; ++s) {
            bar_init(acc_full + 8 * s, 1);
            bar_init(acc_empty + 8 * s, 8 * kTeams);  // the teams' warps in either CTA
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

    if (warp == 0) {
        if (lane == 0) {
            int step = 0;
            bool ok = true;
            for (int i = pair; ok && i < tiles; i += pairs) {
                const Tile t = tile_of(p, i);
                const int am = t.m * kTile + rank * kRowsCta;  // this CTA's rows of A
                // its rows of B: of the gate (first CTA) or the other projection (second), or half the tile's columns
                const int bn = kGated ? t.n * kRowsCta + (int)rank * p.n : t.n * kTile + (int)rank * kRowsCta;
                for (int k = t.k0; k < t.k1; ++k, ++step) {
                    const int s = step % kStages;
                    if (!(ok = bar_wait(empty + 8 * s, (step / kStages & 1) ^ 1, dead)))
                        break;
                    if (rank == 0)
                        bar_expect(full + 8 * s, 4 * kHalf);
                    const uint32_t bar = in_cta(full + 8 * s, 0), a = base + s * 2 * kHalf, b = a + kHalf;
                    // (what rounding left goes first: accumulators are truncated at every addition, small ones by little)
                    const int second = !kGated && k < p.k_once, term = (k - (kGated || second ? 0 : p.k_once)) * kBlockK;
                    if (kARows) {
                        load_box(a, &a_map, am, term, second, bar);
                        load_box(a + kHalf / 2, &a_map, am + 64, term, second, bar);
                    } else if (!kGated) {
                        load_box(a, &a_map, term, am, second, bar);
                    } else {
                        load_box(a, &a_map, term, am, bar);
                    }
                    if (kBRows) {
                        load_box(b, &b_map, bn, term, bar);
                        load_box(b + kHalf / 2, &b_map, bn + 64, term, bar);
                    } else {
                        load_box(b, &b_map, term, bn, bar);
                    }
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            // 32-bit sums, operands bf16 or f16, 256 x 256, each along its terms or its rows
            const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            const uint32_t kind = 1u << 4 | type << 7 | type << 10 | (uint32_t)kARows << 15 | (uint32_t)kBRows << 16 |
                                  (kTile / 8) << 17 | (kTile / 16) << 24;
            int step = 0, done = 0;
            bool ok = true;
            for (int i = pair; ok && i < tiles; i += pairs, ++done) {
                const Tile t = tile_of(p, i);
                const int set = done & 1;
                if (!(ok = bar_wait(acc_empty + 8 * set, (done >> 1 & 1) ^ 1, dead)))
                    break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t acc = tmem + set * kTile;
                for (int k = t.k0; k < t.k1; ++k, ++step) {
                    const int s = step % kStages;
                    if (!(ok = bar_wait(full + 8 * s, step / kStages & 1, dead)))
                        break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = base + s * 2 * kHalf;
                    const uint64_t a = operand<kARows>(at), b = operand<kBRows>(at + kHalf);
#pragma unroll
                    for (int q = 0; q < kBlockK / 16; ++q)  // 16 terms: 32 bytes on, or two groups of eight terms
                        multiply(acc, a + q * (kARows ? 128 : 2), b + q * (kBRows ? 128 : 2), kind, k > t.k0 || q > 0);
                    commit(empty + 8 * s);
                }
                if (ok)
                    commit(acc_full + 8 * set);
            }
        }
    } else {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        const int team = (warp - 2) >> 2;
        const bool first = (threadIdx.x - 64) % 128 == 0;  // issues its team's stores
        const uint32_t slab0 = slabs + team * kSlabs * kSlab;
        const float scale = kScaled<T> && kForm != kForward ? scale_of(p.peaks) : 1.0f, back = 1.0f / scale;
        int done = 0;
        bool ok = true;
        for (int i = pair; i < tiles; i += pairs, ++done) {
            const Tile t = tile_of(p, i);
            const int set = done & 1;
            // (past a wait that ran out the outputs are NaN, so that no wrong result passes for a right one: also those
            // of later tiles, whose products never start, though the barrier shows the parity they wait for)
            ok = __all_sync(~0u, ok && bar_wait(acc_full + 8 * set, done >> 1 & 1, dead));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + set * kTile + ((uint32_t)(quarter * 32) << 16);
            const int m0 = t.m * kTile + rank * kRowsCta;
            auto columns = [&](int c, float (&v)[32]) {
                if (ok) {
                    load_acc(acc + c, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        v[e] = __int_as_float(0x7fffffff);
                }
            };
            if (kForm == kForward) {
                const int c = team * 64;  // 64 columns of H a team
                if (first)
                    stores_left<0>();
                team_sync(team);
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    float g[32], u[32];
                    columns(c + half * 32, g);
                    columns(kRowsCta + c + half * 32, u);
                    wait_acc();
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float f, slope;
                        activate<kAct>(g[e], f, slope);
                        g[e] = f * u[e];
                    }
                    put32<T>(slab0, row, half, g);
                }
                fence_async();
                team_sync(team);
                const int col = t.n * kRowsCta + c;
                if (first && col < p.n && m0 < p.m)
                    store_box(&out_map, slab0, col, 0, m0);
                if (first)
                    stores_close();
            } else if (kForm == kProjGrad) {
#pragma unroll 1
                for (int c = team * 32; c < kRowsCta; c += 32 * kTeams) {  // 32 columns of H, both values of dg and du
                    if (first)
                        stores_left<0>();
                    team_sync(team);
                    const int col = t.n * kRowsCta + c;
                    float g[32], u[32], d[32];
                    columns(c, g);
                    columns(kRowsCta + c, u);
                    const T *dh = (const T *)p.dh + (int64_t)(m0 + row) * p.dhs + col;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint4 q = make_uint4(0, 0, 0, 0);
                        if (m0 + row < p.m && col + e < p.n)
                            q = __ldg(reinterpret_cast<const uint4 *>(dh + e));
                        unpack8<T>(q, d + e);
                    }
                    wait_acc();
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        float f, slope;
                        activate<kAct>(g[e], f, slope);
                        const float up = kScaled<T> ? d[e] * scale : d[e];
                        g[e] = up * u[e] * slope;
                        u[e] = up * f;
                    }
                    put32_in_two<T>(slab0, row, g);
                    put32_in_two<T>(slab0 + kSlab, row, u);
                    fence_async();
                    team_sync(team);
                    if (first && col < p.n && m0 < p.m) {
#pragma unroll
                        for (int k = 0; k < 2 * kValues; ++k)  // dg, du, and what they left
                            store_box(&out_map, slab0 + (k & 1) * kSlab + (k >> 1) * kHalfSlab, col, k, m0);
                    }
                    if (first)
                        stores_close();
                }
            } else {
                constexpr int kWide = kParts ? 32 : 64;  // columns of 128 bytes
#pragma unroll 1
                for (int c = 0; c < kTile; c += kWide) {
                    if (first)
                        stores_left<1>();
                    team_sync(team);
                    const uint32_t slab = slab0 + (c / kWide & 1) * kSlab;
                    float v[32];
                    if (kParts) {
                        columns(c, v);
                        wait_acc();
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            put16(slab, row, q, __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]),
                                  __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
                    } else {
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            columns(c + half * 32, v);
                            wait_acc();
                            if (kScaled<T>) {
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    v[e] *= back;
                            }
                            put32<T>(slab, row, half, v);
                        }
                    }
                    fence_async();
                    team_sync(team);
                    if (first && t.n * kTile + c < p.n && m0 < p.m)
                        store_box(&out_map, slab, t.n * kTile + c, m0, t.split);
                    if (first)
                        stores_close();
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0)
                bar_arrive_cluster(in_cta(acc_empty + 8 * set, 0));
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

// The sum of the parts, brought back from its scale and rounded; parts in order.
template <class T>
__global__ void ffn_parts_kernel(int64_t rows, int64_t cols, int splits, const float *parts, T *out, int64_t os,
                                 Peaks peaks)
{
    const int64_t per = cols / 4, n = rows * per;
    next_may_start();
    after_previous();
    const float back = kScaled<T> ? 1.0f / scale_of(peaks) : 1.0f;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
        float4 v = reinterpret_cast<const float4 *>(parts)[i];
        for (int s = 1; s < splits; ++s) {
            const float4 q = reinterpret_cast<const float4 *>(parts)[i + s * n];
            v.x += q.x, v.y += q.y, v.z += q.z, v.w += q.w;
        }
        if (kScaled<T>)
            v.x *= back, v.y *= back, v.z *= back, v.w *= back;
        *reinterpret_cast<uint2 *>(out + i / per * os + i % per * 4) = make_uint2(pack2<T>(v.x, v.y), pack2<T>(v.z, v.w));
    }
}

// ------------------------------------------------------------ host

// An operand: [rows][cols], boxes of box_rows x 64 columns.
bool operand_map(CUtensorMap *map, int dtype, const void *p, int64_t rows, int64_t cols, int64_t stride, int box_rows)
{
    const int64_t dims[2] = {cols, rows}, strides[1] = {rows > 1 ? stride : cols};
    const int box[2] = {64, box_rows};
    return make_map(map, dtype, p, 2, dims, strides, box);
}

// dg and du as A: [value][row][2 H] by columns, rows and values, boxes of box_rows x 64 columns.
bool grads_map(CUtensorMap *map, int dtype, const void *p, int64_t rows, int64_t H, int box_rows)
{
    const int64_t dims[3] = {2 * H, rows, kValues}, strides[2] = {2 * kValues * H, 2 * H};
    const int box[3] = {64, box_rows, 1};
    return make_map(map, dtype, p, 3, dims, strides, box);
}

constexpr int kPairs = 76;  // of a GB300's 152 SMs

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Into how many parts the terms of a product are dealt: the number that ends
// soonest.  A block of 64 terms takes a pair 0.27 us; each part writes its
// sums in 32 bits, 0.8 us a tile, and a pass adds them up (3 us and 8 bytes a
// sum and part at 5 TB/s).
int splits_for(int64_t m, int64_t n, int64_t blocks)
{
    const int64_t tiles = up(m, kTile) * up(n, kTile);
    int best = 1;
    double least = 0.0;
    for (int s = 1; s <= 16 && s <= blocks; ++s) {
        const double waves = (double)up(tiles * s, kPairs), length = (double)up(blocks, s);
        double us = waves * (0.27 * length + (s > 1 ? 0.8 : 0.4));
        if (s > 1)
            us += 3.0 + (double)m * n * 8 * s / 5e6;
        if (s == 1 || us < least) {
            least = us;
            best = s;
        }
    }
    return best;
}

int64_t parts_bytes(int64_t m, int64_t n, int64_t blocks)
{
    const int s = splits_for(m, n, blocks);
    return s > 1 ? (int64_t)s * m * n * 4 : 0;
}

int64_t dgu_bytes(int64_t rows, int64_t H) { return up(rows * 2 * kValues * H * 2, 256) * 256; }

template <class T, int kForm, int kAct, bool kParts>
cudaError_t go(const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out, const Params &p, cudaStream_t st,
               bool chained)
{
    const auto kernel = ffn_kernel<T, kForm, kAct, kParts>;  // (kAct plays no part in the last two forms)
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(kForm));
    if (e != cudaSuccess)
        return e;
    const int64_t tiles = (int64_t)p.m_tiles * p.n_tiles * p.splits;
    return launch_chained(kernel, 2 * (unsigned)(tiles < kPairs ? tiles : kPairs), threads_of(kForm), smem_of(kForm), st,
                          chained, a, b, out, p);
}

// out [m][n] = A B, A as two values, in one go or in parts.
template <class T, int kForm>
cudaError_t product(int dtype, const CUtensorMap &a, const CUtensorMap &b, int64_t m, int64_t n, int64_t k, void *out,
                    int64_t os, float *parts, Peaks peaks, cudaStream_t st)
{
    Params p{};
    p.peaks = peaks;
    p.m = (int)m;
    p.n = (int)n;
    p.m_tiles = (int)up(m, kTile);
    p.n_tiles = (int)up(n, kTile);
    p.k_once = (int)up(k, kBlockK);
    p.k_blocks = kValues * p.k_once;
    p.splits = splits_for(m, n, p.k_blocks);
    CUtensorMap map;
    const int64_t dims[3] = {n, m, p.splits};
    if (p.splits == 1) {
        const int64_t strides[2] = {m > 1 ? os : n, (m > 1 ? os : n) * m};
        const int box[3] = {64, kRowsCta, 1};
        if (!make_map(&map, dtype, out, 3, dims, strides, box))
            return cudaErrorInvalidValue;
        return go<T, kForm, AV_SILU, false>(a, b, map, p, st, true);
    }
    const int64_t strides[2] = {n, m * n};
    const int box[3] = {32, kRowsCta, 1};
    if (!make_map(&map, AV_F32, parts, 3, dims, strides, box))
        return cudaErrorInvalidValue;
    cudaError_t e = go<T, kForm, AV_SILU, true>(a, b, map, p, st, true);
    if (e != cudaSuccess)
        return e;
    const int64_t blocks = up(m * n / 4, 256);
    return launch_chained(ffn_parts_kernel<T>, (unsigned)(blocks < 152 * 8 ? blocks : 152 * 8), 256, 0, st, true, m, n,
                          p.splits, parts, (T *)out, m > 1 ? os : n, peaks);
}

template <class T, int kAct, bool kGrad>
void few(int rows, int64_t D, int64_t H, const T *x, int64_t xs, const T *w, T *h, int64_t hs, const T *dh, int64_t dhs,
         T *dgu, Peaks peaks, cudaStream_t st)
{
    const unsigned grid = (unsigned)up(H, kFewThreads / 32);
    if (rows <= 1)
        ffn_few_kernel<T, kAct, 1, kGrad><<<grid, kFewThreads, 0, st>>>(rows, D, H, x, xs, w, h, hs, dh, dhs, dgu, peaks);
    else
        ffn_few_kernel<T, kAct, kFewRows, kGrad><<<grid, kFewThreads, 0, st>>>(rows, D, H, x, xs, w, h, hs, dh, dhs, dgu, peaks);
}

// h, or the projections' gradients [rows][value][2][H].
template <class T, int kAct, bool kGrad>
cudaError_t gated(int dtype, int64_t rows, int64_t D, int64_t H, const void *x, int64_t xs, const void *w, void *h,
                  int64_t hs, const void *dh, int64_t dhs, void *dgu, Peaks peaks, cudaStream_t st)
{
    if (rows <= kFewRows) {
        few<T, kAct, kGrad>((int)rows, D, H, (const T *)x, xs, (const T *)w, (T *)h, hs, (const T *)dh, dhs, (T *)dgu,
                            peaks, st);
        return cudaGetLastError();
    }
    Params p{};
    p.m = (int)rows;
    p.n = (int)H;
    p.m_tiles = (int)up(rows, kTile);
    p.n_tiles = (int)up(H, kRowsCta);
    p.k_blocks = (int)up(D, kBlockK);
    p.k_once = p.k_blocks;
    p.splits = 1;
    p.dh = dh;
    p.dhs = dhs;
    p.peaks = peaks;
    CUtensorMap a, b, out;
    // (stores are columns, projection of a value, row; h has one)
    const int64_t dims[3] = {H, kGrad ? 2 * kValues : 1, rows}, strides[2] = {H, kGrad ? 2 * kValues * H : hs};
    const int box[3] = {kGrad ? 32 : 64, 1, kRowsCta};
    if (!operand_map(&a, dtype, x, rows, D, xs, kRowsCta) || !operand_map(&b, dtype, w, 2 * H, D, D, kRowsCta) ||
        !make_map(&out, dtype, kGrad ? dgu : h, 3, dims, strides, box, kGrad ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    return go<T, kGrad ? kProjGrad : kForward, kAct, false>(a, b, out, p, st, false);
}

}  // namespace

int64_t ffn_work_bytes(int64_t rows, int64_t D, int64_t H)
{
    const int64_t a = parts_bytes(rows, D, kValues * up(2 * H, kBlockK)),
                  b = parts_bytes(2 * H, D, kValues * up(rows, kBlockK));
    return dgu_bytes(rows, H) + (a > b ? a : b) + kPeakBytes;  // (the peaks last)
}

cudaError_t launch_ffn(int64_t rows, int64_t D, int64_t H, int dtype, int act, const void *x, int64_t x_stride,
                       const void *w, void *h, int64_t h_stride, cudaStream_t st)
{
    if (!map_encoder())
        return cudaErrorNotSupported;
    auto run = [&](auto v) {
        using T = decltype(v);
        return act == AV_SILU ? gated<T, AV_SILU, false>(dtype, rows, D, H, x, x_stride, w, h, h_stride, nullptr, 0,
                                                         nullptr, nullptr, st)
                              : gated<T, AV_GELU, false>(dtype, rows, D, H, x, x_stride, w, h, h_stride, nullptr, 0,
                                                         nullptr, nullptr, st);
    };
    return dtype == AV_BF16 ? run(__nv_bfloat16()) : run(__half());
}

cudaError_t launch_ffn_grad(int64_t rows, int64_t D, int64_t H, int dtype, int act, const void *dh, int64_t dh_stride,
                            const void *x, int64_t x_stride, const void *w, void *dx, int64_t dx_stride, void *dw,
                            void *work, cudaStream_t st)
{
    if (!map_encoder())
        return cudaErrorNotSupported;
    float *parts = reinterpret_cast<float *>((char *)work + dgu_bytes(rows, H));
    float4 *peaks = reinterpret_cast<float4 *>((char *)work + ffn_work_bytes(rows, D, H) - kPeakBytes);
    auto run = [&](auto v) {
        using T = decltype(v);
        cudaError_t e = cudaSuccess;
        if constexpr (kScaled<T>) {
            e = cudaMemsetAsync(peaks, 0, kPeakBytes, st);
            if (e != cudaSuccess)
                return e;
            const int64_t blocks = up(rows > 2 * H ? rows : 2 * H, kPeakThreads / 32);
            ffn_peaks_kernel<T><<<dim3((unsigned)(blocks < 152 * 8 ? blocks : 152 * 8), 3), kPeakThreads, 0, st>>>(
                rows, D, H, (const T *)x, x_stride, (const T *)w, (const T *)dh, dh_stride, peaks);
        }
        e = act == AV_SILU ? gated<T, AV_SILU, true>(dtype, rows, D, H, x, x_stride, w, nullptr, 0, dh,
                                                                 dh_stride, work, peaks, st)
                                       : gated<T, AV_GELU, true>(dtype, rows, D, H, x, x_stride, w, nullptr, 0, dh,
                                                                 dh_stride, work, peaks, st);
        if (e != cudaSuccess)
            return e;
        CUtensorMap dgu, wt, dgut, xt;
        if (!grads_map(&dgu, dtype, work, rows, H, kRowsCta) || !operand_map(&wt, dtype, w, 2 * H, D, D, 64) ||
            !grads_map(&dgut, dtype, work, rows, H, 64) || !operand_map(&xt, dtype, x, rows, D, x_stride, 64))
            return cudaErrorInvalidValue;
        e = product<T, kTimesW>(dtype, dgu, wt, rows, D, 2 * H, dx, dx_stride, parts, peaks, st);
        if (e != cudaSuccess)
            return e;
        return product<T, kTransposed>(dtype, dgut, xt, 2 * H, D, rows, dw, D, parts, peaks, st);
    };
    return dtype == AV_BF16 ? run(__nv_bfloat16()) : run(__half());
}

}  // namespace av
