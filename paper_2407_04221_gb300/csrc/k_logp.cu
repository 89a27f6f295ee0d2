// k_logp.cu -- log probabilities of given tokens, entropy, top alternatives,
// and the gradient.  With m the row's largest logit and e_j = exp(x_j - m):
//   logz = log sum e,  log p_j = (x_j - m) - logz,  entropy = logz - sum e (x - m) / sum e
//   dx_j = dlogp (1[j = token] - p_j) - dentropy p_j (log p_j + entropy)
//
// Forward, the logits are read once: every thread keeps a running maximum with
// the sums below it, brought to a new maximum when one comes, and the threads'
// sums are joined at the row's.  Bound by memory, for 16-bit logits nearly by
// the exponentials (one an entry: 16 of an SM's 128 lanes).
//
// The k largest: the k-th largest of the threads' maxima is no larger than the
// k-th largest entry, so only threads whose maximum reaches it look at their
// entries again, and only entries that reach it are listed: k and a few.  Their
// order is counted out by (value, lowest index).  Should the list run over
// (rows of equal values), the k largest are drawn one by one instead.
//
// Rows of up to 32 entries take a thread, up to 1,024 a warp, else a block.
// Addition has one order throughout: equal rows give equal bits.
#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kTiny = 32;          // entries of a row that a thread takes
constexpr int kTinyThreads = 128;
constexpr int kNarrow = 1024;      // entries of a row that a warp takes
constexpr int kNarrowThreads = 256;
constexpr int kWideThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.402823466e38f;

__device__ __forceinline__ float no_value() { return -INFINITY; }

__device__ __forceinline__ int64_t token_of(const void *tokens, int bytes, int64_t r)
{
    return bytes == 1 ? ((const uint8_t *)tokens)[r] : bytes == 4 ? ((const int32_t *)tokens)[r]
                                                                  : ((const int64_t *)tokens)[r];
}

__device__ __forceinline__ float exp2_fast(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The larger; NaN where either is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// exp(d) for d <= 0, and d kept finite for products: exp is 0 from -104 on.
__device__ __forceinline__ float exp_below(float &d)
{
    d = max_nan(d, -200.0f);
    return exp2_fast(d * kLog2e);
}

// A value as a whole number of the same order, NaN above all, both zeros
// alike; an entry that is not there (-inf) is 0.
__device__ __forceinline__ uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.0f);
    if (x != x)
        return 0xffffffffu;
    return x == no_value() ? 0u : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// (value, index): larger values first, then lower indices; 0 is no entry.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t j)
{
    const uint32_t u = order_of(x);
    return u ? (uint64_t)u << 32 | (uint32_t)~j : 0;
}

// The running maximum and the sums of exp(x - m) and exp(x - m) (x - m).
struct Sums {
    float m, e, ex;
    uint32_t top;  // order_of the largest, NaN included
};

__device__ __forceinline__ void raise(Sums &s, float m)
{
    const float d = s.m - m;  // (-inf where an infinite logit comes: the sums are NaN from there on, or 0)
    float c = d;
    const float k = exp_below(c);
    s.ex = k * (s.ex + s.e * c);
    s.e *= k;
    s.m = m;
}

__device__ __forceinline__ void add(Sums &s, float x)
{
    float d = x - s.m;
    const float p = exp_below(d);
    s.e += p;
    s.ex = fmaf(p, d, s.ex);
}

// kN entries at a time.
template <bool kTop, int kN>
__device__ __forceinline__ void take(Sums &s, const float (&x)[kN])
{
    float m = x[0];
#pragma unroll
    for (int k = 1; k < kN; ++k)
        m = fmaxf(m, x[k]);
    if (m > s.m)
        raise(s, m);
#pragma unroll
    for (int k = 0; k < kN; ++k)
        add(s, x[k]);
    if (kTop) {
        bool bad = false;
#pragma unroll
        for (int k = 0; k < kN; ++k)
            bad |= x[k] != x[k];
        const uint32_t u = bad ? 0xffffffffu : order_of(m);
        s.top = u > s.top ? u : s.top;
    }
}

// A row of logits seen in packs of 16 bytes: entries before the first boundary,
// packs, entries after the last.
template <class T>
struct Row {
    static constexpr int kPack = 16 / sizeof(T);
    const T *x;
    const uint8_t *mask;
    int V, head, packs;

    __device__ __forceinline__ Row(const T *row, const uint8_t *m, int n) : x(row), mask(m), V(n)
    {
        head = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int)sizeof(T);
        head = head < V ? head : V;
        packs = (V - head) / kPack;
    }
    // entries outside the packs, and the place of the i-th
    __device__ __forceinline__ int loose() const { return V - packs * kPack; }
    __device__ __forceinline__ int loose_at(int i) const { return i < head ? i : i + packs * kPack; }
    template <bool kMask>
    __device__ __forceinline__ float entry(int j) const
    {
        return kMask && mask[j] == 0 ? no_value() : to_f32(x[j]);
    }
    __device__ __forceinline__ uint4 raw(int i) const { return *reinterpret_cast<const uint4 *>(x + head + i * kPack); }
    template <bool kMask>
    __device__ __forceinline__ void open(uint4 q, int i, float (&v)[kPack]) const
    {
        const T *p = reinterpret_cast<const T *>(&q);
#pragma unroll
        for (int k = 0; k < kPack; ++k)
            v[k] = kMask && mask[head + i * kPack + k] == 0 ? no_value() : to_f32(p[k]);
    }
};

// All threads of the row: a warp, or the block.
template <int kGroup>
__device__ __forceinline__ void group_sync()
{
    if (kGroup == 32)
        __syncwarp();
    else
        __syncthreads();
}

template <int kGroup, class F>
__device__ __forceinline__ float reduce(float v, float *slots, F f)
{
#pragma unroll
    for (int o = 16; o; o >>= 1)
        v = f(v, __shfl_xor_sync(~0u, v, o));
    if (kGroup == 32)
        return v;
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = slots[threadIdx.x & (kGroup / 32 - 1)];
#pragma unroll
    for (int o = kGroup / 64; o; o >>= 1)
        v = f(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

constexpr int kListed = 512;  // candidates of a block's row, and of a warp's:
constexpr int kListedWarp = 96;

template <int kGroup>
struct Scratch {
    static constexpr int kWarps = kGroup / 32;
    float slots[kWarps];
    uint32_t heads[kWarps * AV_MAX_TOP];
    uint32_t floor;
    int count;
    uint64_t best[kWarps];
    uint64_t list[kGroup == 32 ? kListedWarp : kListed];
};

// The k-th largest of the threads' values (0 where there are fewer).
template <int kGroup>
__device__ uint32_t kth(uint32_t v, int k, Scratch<kGroup> &s)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t last = 0;
    for (int i = 0; i < k; ++i) {
        last = __reduce_max_sync(~0u, v);
        const uint32_t holders = __ballot_sync(~0u, v == last);
        if (lane == __ffs(holders) - 1)
            v = 0;
        if (kGroup > 32 && lane == 0)
            s.heads[warp * AV_MAX_TOP + i] = last;
    }
    if (kGroup == 32)
        return last;
    __syncthreads();
    if (warp == 0) {  // each warp's are in order: a lane holds the next of one
        int at = 0;
        for (int i = 0; i < k; ++i) {
            const uint32_t u = lane < kGroup / 32 && at < k ? s.heads[lane * AV_MAX_TOP + at] : 0;
            last = __reduce_max_sync(~0u, u);
            const uint32_t holders = __ballot_sync(~0u, u == last && lane < kGroup / 32);
            at += lane == __ffs(holders) - 1;
        }
        if (lane == 0)
            s.floor = last;
    }
    __syncthreads();
    return s.floor;
}

// f(value, index) for this thread's entries of the row.
template <int kGroup, bool kMask, class T, class F>
__device__ __forceinline__ void entries(const Row<T> &row, int thread, F f)
{
    for (int i = thread; i < row.loose(); i += kGroup)
        f(row.template entry<kMask>(row.loose_at(i)), row.loose_at(i));
    for (int i = thread; i < row.packs; i += kGroup) {
        float v[Row<T>::kPack];
        row.template open<kMask>(row.raw(i), i, v);
#pragma unroll
        for (int k = 0; k < Row<T>::kPack; ++k)
            f(v[k], row.head + i * Row<T>::kPack + k);
    }
}

template <class T, int kGroup, int kThreads, bool kMask, bool kTop>
__global__ __launch_bounds__(kThreads) void logp_kernel(const LogpArgs a, int top, float *logp, float *entropy,
                                                        float *peak, float *logz, float *top_logp, int32_t *top_index)
{
    constexpr int kPack = Row<T>::kPack, kAhead = 4;
    __shared__ Scratch<kGroup> scratch[kThreads / kGroup];
    Scratch<kGroup> &s = scratch[threadIdx.x / kGroup];
    const int thread = threadIdx.x % kGroup;
    const int64_t groups = (int64_t)gridDim.x * (kThreads / kGroup);
    for (int64_t r = (int64_t)blockIdx.x * (kThreads / kGroup) + threadIdx.x / kGroup; r < a.rows; r += groups) {
        const Row<T> row((const T *)a.logits + r * a.stride, kMask ? a.mask + r * a.mask_stride : nullptr, a.V);
        Sums q{kLowest, 0.0f, 0.0f, 0u};
        int i = thread;
        for (; i + (kAhead - 1) * kGroup < row.packs; i += kAhead * kGroup) {
            uint4 raw[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                raw[k] = row.raw(i + k * kGroup);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                float v[kPack];
                row.template open<kMask>(raw[k], i + k * kGroup, v);
                take<kTop>(q, v);
            }
        }
        for (; i < row.packs; i += kGroup) {
            float v[kPack];
            row.template open<kMask>(row.raw(i), i, v);
            take<kTop>(q, v);
        }
        for (int j = thread; j < row.loose(); j += kGroup) {
            const float v[1] = {row.template entry<kMask>(row.loose_at(j))};
            take<kTop>(q, v);
        }
        const float m = reduce<kGroup>(q.m, s.slots, [](float x, float y) { return fmaxf(x, y); });
        raise(q, m);
        auto plus = [](float x, float y) { return x + y; };
        const float e = reduce<kGroup>(q.e, s.slots, plus), ex = reduce<kGroup>(q.ex, s.slots, plus);
        const bool some = e != 0.0f;  // (NaN counts)
        const float z = some ? logf(e) : no_value();
        if (thread == 0) {
            const int64_t tok = token_of(a.tokens, a.token_bytes, r);
            float lp = 0.0f;
            if (tok >= 0 && tok < a.V) {
                const float x = row.template entry<kMask>((int)tok);
                lp = some ? (x - m) - z : no_value();
            }
            logp[r] = lp;
            if (entropy)
                entropy[r] = some ? z - ex / e : 0.0f;
            if (peak)
                peak[r] = some ? m : no_value();
            if (logz)
                logz[r] = z;
        }
        if (!kTop)
            continue;
        const uint32_t floor = kth<kGroup>(q.top, top, s);
        if (thread == 0)
            s.count = 0;
        group_sync<kGroup>();
        constexpr int kRoom = kGroup == 32 ? kListedWarp : kListed;
        if (q.top >= floor && q.top != 0) {
            entries<kGroup, kMask>(row, thread, [&](float v, int j) {
                const uint32_t u = order_of(v);
                if (u >= floor && u != 0) {
                    const int at = atomicAdd(&s.count, 1);
                    if (at < kRoom)
                        s.list[at] = rank_key(v, j);
                }
            });
        }
        group_sync<kGroup>();
        const int count = s.count;
        if (count <= kRoom) {
            for (int c = thread; c < count; c += kGroup) {
                const uint64_t mine = s.list[c];
                int rank = 0;
                for (int o = 0; o < count; ++o)
                    rank += s.list[o] > mine;
                if (rank < top) {
                    const int j = (int)~(uint32_t)mine;
                    top_index[r * top + rank] = j;
                    top_logp[r * top + rank] = (to_f32(row.x[j]) - m) - z;
                }
            }
            for (int k = count + thread; k < top; k += kGroup) {  // fewer than asked for
                top_index[r * top + k] = -1;
                top_logp[r * top + k] = no_value();
            }
        } else {
            uint64_t last = ~0ull;
            for (int k = 0; k < top; ++k) {
                uint64_t best = 0;
                entries<kGroup, kMask>(row, thread, [&](float v, int j) {
                    const uint64_t key = rank_key(v, j);
                    best = key < last && key > best ? key : best;
                });
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    const uint64_t u = __shfl_xor_sync(~0u, best, o);
                    best = u > best ? u : best;
                }
                if (kGroup > 32) {
                    __syncthreads();
                    if ((threadIdx.x & 31) == 0)
                        s.best[threadIdx.x >> 5] = best;
                    __syncthreads();
                    for (int w = 0; w < kGroup / 32; ++w)
                        best = s.best[w] > best ? s.best[w] : best;
                }
                last = best;
                if (thread == 0) {
                    const int j = (int)~(uint32_t)best;
                    top_index[r * top + k] = best ? j : -1;
                    top_logp[r * top + k] = best ? (to_f32(row.x[j]) - m) - z : no_value();
                }
            }
        }
        group_sync<kGroup>();  // (the list is the next row's)
    }
}

// A thread a row of at most kMost entries, all in registers.
template <class T, int kMost, bool kMask>
__global__ __launch_bounds__(kTinyThreads) void logp_tiny_kernel(const LogpArgs a, int top, float *logp, float *entropy,
                                                                 float *peak, float *logz, float *top_logp,
                                                                 int32_t *top_index)
{
    const int64_t r = (int64_t)blockIdx.x * kTinyThreads + threadIdx.x;
    if (r >= a.rows)
        return;
    const T *x = (const T *)a.logits + r * a.stride;
    const uint8_t *mask = kMask ? a.mask + r * a.mask_stride : nullptr;
    float v[kMost], m = kLowest;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        v[j] = j < a.V && (!kMask || mask[j] != 0) ? to_f32(x[j]) : no_value();
        m = fmaxf(m, v[j]);
    }
    Sums q{m, 0.0f, 0.0f, 0u};
    const int64_t tok = token_of(a.tokens, a.token_bytes, r);
    float given = no_value();
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        if (j < a.V)
            add(q, v[j]);
        given = j == tok ? v[j] : given;
    }
    const bool some = q.e != 0.0f;
    const float z = some ? logf(q.e) : no_value();
    logp[r] = tok >= 0 && tok < a.V ? (some ? (given - m) - z : no_value()) : 0.0f;
    if (entropy)
        entropy[r] = some ? z - q.ex / q.e : 0.0f;
    if (peak)
        peak[r] = some ? m : no_value();
    if (logz)
        logz[r] = z;
    uint32_t gone = 0;
    for (int k = 0; k < top; ++k) {
        uint32_t best = 0;
        int at = -1;
        float value = no_value();
#pragma unroll
        for (int j = 0; j < kMost; ++j) {
            const uint32_t u = gone >> j & 1 ? 0 : order_of(v[j]);
            if (u > best) {
                best = u;
                at = j;
                value = v[j];
            }
        }
        gone |= at >= 0 ? 1u << at : 0;
        top_index[r * top + k] = at;
        top_logp[r * top + k] = at >= 0 ? (value - m) - z : no_value();
    }
}

// What a row's gradient takes; c and de 2^-24 of what they are.
struct Slope {
    float m, z, dl, c, de;
    int64_t tok;
    bool some;
};
__device__ __forceinline__ Slope slope_of(const LogpArgs &a, int64_t r, const float *dlogp, const float *dentropy,
                                          const float *peak, const float *logz, const float *entropy)
{
    Slope s;
    s.m = peak[r];
    s.z = logz[r];
    s.some = s.z != no_value();
    s.de = dentropy ? dentropy[r] : 0.0f;
    s.tok = token_of(a.tokens, a.token_bytes, r);
    s.dl = dlogp && s.tok >= 0 && s.tok < a.V ? dlogp[r] : 0.0f;
    s.c = (s.dl + s.de * (dentropy ? entropy[r] : 0.0f)) * 0x1p-24f;
    s.de *= 0x1p-24f;
    return s;
}

// Of an entry (-inf where it is masked), but for the token's own dlogp.  The
// exponential is taken 2^24 times too large: it flushes to 0 at 2^-126, where
// its product with a log probability does not yet.
__device__ __forceinline__ float slope_at(const Slope &s, float x)
{
    const float lp = max_nan((x - s.m) - s.z, -200.0f);
    const float p = exp2_fast(fmaf(lp, kLog2e, 24.0f));
    return -p * fmaf(s.de, lp, s.c);
}

// A block (or a warp) takes a row, or with gridDim.y a part of it.
template <class T, int kGroup, int kThreads, bool kMask>
__global__ __launch_bounds__(kThreads) void logp_grad_kernel(const LogpArgs a, const float *dlogp,
                                                             const float *dentropy, const float *peak,
                                                             const float *logz, const float *entropy, T *dlogits,
                                                             int64_t dstride, bool packed)
{
    constexpr int kPack = Row<T>::kPack, kAhead = 4;
    const int64_t r = (int64_t)blockIdx.x * (kThreads / kGroup) + threadIdx.x / kGroup;
    if (r >= a.rows)
        return;
    const Row<T> row((const T *)a.logits + r * a.stride, kMask ? a.mask + r * a.mask_stride : nullptr, a.V);
    const Slope s = slope_of(a, r, dlogp, dentropy, peak, logz, entropy);
    T *dx = dlogits + r * dstride;
    const int thread = threadIdx.x % kGroup + blockIdx.y * kGroup, step = kGroup * gridDim.y;
    auto value = [&](float x, int j) {
        if (!s.some || (kMask && x == no_value()))
            return 0.0f;
        return slope_at(s, x) + (j == s.tok && x != no_value() ? s.dl : 0.0f);
    };
    if (!packed) {  // dlogits' rows begin elsewhere in 16 bytes than those of logits
        for (int j = thread; j < a.V; j += step)
            dx[j] = from_f32<T>(value(row.template entry<kMask>(j), j));
        return;
    }
    for (int i = thread; i < row.loose(); i += step) {
        const int j = row.loose_at(i);
        dx[j] = from_f32<T>(value(row.template entry<kMask>(j), j));
    }
    for (int i0 = thread; i0 < row.packs; i0 += kAhead * step) {
        uint4 raw[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            raw[k] = i0 + k * step < row.packs ? row.raw(i0 + k * step) : uint4{};
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = i0 + k * step;
            if (i >= row.packs)
                break;
            float v[kPack];
            row.template open<kMask>(raw[k], i, v);
            uint4 out;
            T *o = reinterpret_cast<T *>(&out);
            const int j = row.head + i * kPack;
            if (!kMask && s.some && (s.tok < j || s.tok >= j + kPack)) {
#pragma unroll
                for (int e = 0; e < kPack; ++e)
                    o[e] = from_f32<T>(slope_at(s, v[e]));
            } else {
#pragma unroll
                for (int e = 0; e < kPack; ++e)
                    o[e] = from_f32<T>(value(v[e], j + e));
            }
            *reinterpret_cast<uint4 *>(dx + j) = out;
        }
    }
}

template <class T, bool kMask>
__global__ __launch_bounds__(kTinyThreads) void logp_grad_tiny_kernel(const LogpArgs a, const float *dlogp,
                                                                      const float *dentropy, const float *peak,
                                                                      const float *logz, const float *entropy,
                                                                      T *dlogits, int64_t dstride)
{
    const int64_t r = (int64_t)blockIdx.x * kTinyThreads + threadIdx.x;
    if (r >= a.rows)
        return;
    const T *x = (const T *)a.logits + r * a.stride;
    const Slope s = slope_of(a, r, dlogp, dentropy, peak, logz, entropy);
#pragma unroll 8
    for (int j = 0; j < a.V; ++j) {
        const float v = kMask && a.mask[r * a.mask_stride + j] == 0 ? no_value() : to_f32(x[j]);
        const float g = !s.some || (kMask && v == no_value())
                            ? 0.0f
                            : slope_at(s, v) + (j == s.tok && v != no_value() ? s.dl : 0.0f);
        dlogits[r * dstride + j] = from_f32<T>(g);
    }
}

// ------------------------------------------------------------ host

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <class F>
void with_flag(bool v, F f)
{
    if (v)
        f(std::true_type());
    else
        f(std::false_type());
}

}  // namespace

cudaError_t launch_logp(const LogpArgs &a, int top, float *logp, float *entropy, float *peak, float *logz,
                        float *top_logp, int32_t *top_index, cudaStream_t st)
{
    with_type(a.dtype, [&](auto v) {
        using T = decltype(v);
        with_flag(a.mask != nullptr, [&](auto mask) {
            if (a.V <= kTiny) {
                auto run = [&](auto kernel) {
                    kernel<<<(unsigned)up(a.rows, kTinyThreads), kTinyThreads, 0, st>>>(a, top, logp, entropy, peak,
                                                                                        logz, top_logp, top_index);
                };
                if (a.V <= 8)
                    run(logp_tiny_kernel<T, 8, mask.value>);
                else
                    run(logp_tiny_kernel<T, kTiny, mask.value>);
                return;
            }
            with_flag(top > 0, [&](auto tops) {
                if (a.V <= kNarrow) {
                    const int64_t blocks = up(a.rows, kNarrowThreads / 32), most = 152 * 8 * 4;
                    logp_kernel<T, 32, kNarrowThreads, mask.value, tops.value>
                        <<<(unsigned)(blocks < most ? blocks : most), kNarrowThreads, 0, st>>>(
                            a, top, logp, entropy, peak, logz, top_logp, top_index);
                } else {
                    const int64_t most = 152 * 4 * 4;
                    logp_kernel<T, kWideThreads, kWideThreads, mask.value, tops.value>
                        <<<(unsigned)(a.rows < most ? a.rows : most), kWideThreads, 0, st>>>(
                            a, top, logp, entropy, peak, logz, top_logp, top_index);
                }
            });
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_logp_grad(const LogpArgs &a, const float *dlogp, const float *dentropy, const float *peak,
                             const float *logz, const float *entropy, void *dlogits, int64_t dlogit_stride,
                             cudaStream_t st)
{
    with_type(a.dtype, [&](auto v) {
        using T = decltype(v);
        T *dx = (T *)dlogits;
        const int64_t e = sizeof(T);
        const bool packed = ((reinterpret_cast<uintptr_t>(dlogits) ^ reinterpret_cast<uintptr_t>(a.logits)) & 15) == 0 &&
                            (a.rows <= 1 || (dlogit_stride - a.stride) * e % 16 == 0);
        with_flag(a.mask != nullptr, [&](auto mask) {
            if (a.V <= kTiny) {
                logp_grad_tiny_kernel<T, mask.value><<<(unsigned)up(a.rows, kTinyThreads), kTinyThreads, 0, st>>>(
                    a, dlogp, dentropy, peak, logz, entropy, dx, dlogit_stride);
            } else if (a.V <= kNarrow) {
                logp_grad_kernel<T, 32, kNarrowThreads, mask.value>
                    <<<(unsigned)up(a.rows, kNarrowThreads / 32), kNarrowThreads, 0, st>>>(
                        a, dlogp, dentropy, peak, logz, entropy, dx, dlogit_stride, packed);
            } else {
                const int parts = (int)up(a.V, 16384);  // (of a row; blocks of some 16,384 entries)
                logp_grad_kernel<T, kNarrowThreads, kNarrowThreads, mask.value>
                    <<<dim3((unsigned)a.rows, (unsigned)(parts < 65535 ? parts : 65535)), kNarrowThreads, 0, st>>>(
                        a, dlogp, dentropy, peak, logz, entropy, dx, dlogit_stride, packed);
            }
        });
    });
    return cudaGetLastError();
}

}  // namespace av
