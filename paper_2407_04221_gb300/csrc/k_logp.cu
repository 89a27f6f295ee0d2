// k_logp.cu -- log probabilities of given tokens, entropy, top alternatives,
// and the gradient.  With m the row's largest logit and e_j = exp(x_j - m):
//   logz = log sum e,  log p_j = (x_j - m) - logz,  entropy = logz - sum e (x - m) / sum e
//   dx_j = dlogp (1[j = token] - p_j) - dentropy p_j (log p_j + entropy)
//
// Forward, the logits are read once.  Rows of up to eight entries take a
// thread, rows of up to 1,024 a group of 2 to 32 lanes that holds them in
// registers, 16 (32) entries a lane.  Longer rows take a block: every thread
// keeps a running maximum with the sums below it, brought to a new maximum when
// one comes, and the threads' sums are joined at the row's.  Bound by memory,
// for 16-bit logits nearly by issue: six instructions an entry.
//
// The k largest of a row in registers are drawn one by one: each lane knows its
// largest, and only the lane that gave one up looks for the next (of 16 bits by
// value and index in one word: 65,536 rows of 256 with eight 49 us, with the
// index apart 78).  Where a warp or a block holds the row they are listed
// instead, in a warp from two on (65,536 rows of 1,000 with four 100 us, drawn
// 154; with twenty 125 and 514; with one 98 and 94): the k-th largest of the
// threads' maxima is no larger than the k-th largest entry, so only entries that
// reach it can be among them, k and a few, and their order is counted out by
// (value, lowest index).  A block looks again only at threads whose maximum
// reaches it, by whole warps.  Should the list run over (rows of equal values),
// or in a block hold NaN, the k largest are drawn one by one all the same.
//
// Addition has one order throughout: equal rows give equal bits.
#include <string.h>

#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kTiny = 8;           // entries of a row that a thread takes
constexpr int kTinyThreads = 128;
constexpr int kNarrow = 1024;      // entries of a row that a group of lanes takes
constexpr int kNarrowThreads = 256;
constexpr int kShort = 64;         // entries of a warp's list of alternatives
constexpr int kGradThreads = 256;
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

// And back.
__device__ __forceinline__ float value_of(uint32_t u)
{
    return u == 0xffffffffu ? __uint_as_float(0x7fffffffu) : __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

// The same of a 16-bit entry in 32 bits, for indices below 65,536.
template <class T>
__device__ __forceinline__ uint32_t short_key(float x, uint32_t j)
{
    if (x == no_value())
        return 0;
    const T t = from_f32<T>(x + 0.0f);  // (as it was read)
    uint16_t b;
    memcpy(&b, &t, 2);
    const uint32_t u = x != x ? 0xffffu : (b & 0x8000u) ? ~(uint32_t)b & 0xffffu : b | 0x8000u;
    return u << 16 | (~j & 0xffffu);
}
template <class T>
__device__ __forceinline__ float short_value(uint32_t key)
{
    const uint32_t u = key >> 16;
    const uint16_t b = (uint16_t)(u & 0x8000u ? u ^ 0x8000u : ~u);
    T t;
    memcpy(&t, &b, 2);
    return u == 0xffffu ? __uint_as_float(0x7fffffffu) : to_f32(t);
}

// The running maximum and the sums of exp(x - m) and exp(x - m) (x - m).
struct Sums {
    float m;
    float2 e, ex;
};

__device__ __forceinline__ void raise(Sums &s, float m)
{
    float d = s.m - m;  // (-inf where an infinite logit comes: the sums are NaN from there on, or 0)
    const float k = exp_below(d);
    const float2 k2 = make_float2(k, k);
    s.ex = mul2(k2, fma2(s.e, make_float2(d, d), s.ex));
    s.e = mul2(s.e, k2);
    s.m = m;
}

// Two entries, none above the maximum.
__device__ __forceinline__ void add(Sums &s, float2 x)
{
    float2 d = add2(x, make_float2(-s.m, -s.m));
    d.x = max_nan(d.x, -200.0f);
    d.y = max_nan(d.y, -200.0f);
    const float2 t = mul2(d, make_float2(kLog2e, kLog2e)), p = make_float2(exp2_fast(t.x), exp2_fast(t.y));
    s.e = add2(s.e, p);
    s.ex = fma2(p, d, s.ex);
}

// kN entries at a time.
template <int kN>
__device__ __forceinline__ void take(Sums &s, const float (&x)[kN])
{
    float m = x[0];
#pragma unroll
    for (int k = 1; k < kN; ++k)
        m = fmaxf(m, x[k]);
    if (m > s.m)
        raise(s, m);
#pragma unroll
    for (int k = 0; k < kN; k += 2)
        add(s, make_float2(x[k], k + 1 < kN ? x[k + 1] : no_value()));
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

template <int kWideThreads, class F>
__device__ __forceinline__ float reduce(float v, float *slots, F f)
{
#pragma unroll
    for (int o = 16; o; o >>= 1)
        v = f(v, __shfl_xor_sync(~0u, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = slots[threadIdx.x & (kWideThreads / 32 - 1)];
#pragma unroll
    for (int o = kWideThreads / 64; o; o >>= 1)
        v = f(v, __shfl_xor_sync(~0u, v, o));
    return v;
}

constexpr int kListed = 512;  // candidates of a row

template <int kWideThreads>
struct Scratch {
    static constexpr int kWarps = kWideThreads / 32;
    float slots[kWarps];
    uint32_t heads[kWarps * AV_MAX_TOP];
    uint32_t floor;
    int count;
    uint64_t best[kWarps];
    uint64_t list[kListed];
};

// The k-th largest of the threads' values.
template <int kWideThreads>
__device__ uint32_t kth(uint32_t v, int k, Scratch<kWideThreads> &s)
{
    constexpr int kWarps = kWideThreads / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t last = 0;
    for (int i = 0; i < k; ++i) {
        last = __reduce_max_sync(~0u, v);
        const uint32_t holders = __ballot_sync(~0u, v == last);
        if (lane == __ffs(holders) - 1)
            v = 0;
        if (lane == 0)
            s.heads[warp * AV_MAX_TOP + i] = last;
    }
    __syncthreads();
    if (warp == 0) {  // each warp's are in order: a lane holds the next of one
        int at = 0;
        for (int i = 0; i < k; ++i) {
            const uint32_t u = lane < kWarps && at < k ? s.heads[lane * AV_MAX_TOP + at] : 0;
            last = __reduce_max_sync(~0u, u);
            const uint32_t holders = __ballot_sync(~0u, u == last && lane < kWarps);
            at += lane == __ffs(holders) - 1;
        }
        if (lane == 0) {
            s.floor = last;
            s.count = 0;
        }
    }
    __syncthreads();
    return s.floor;
}

// f(value, index) for the entries of the row that `thread` takes, seen by
// thread `lane` of `lanes`.
template <int kWideThreads, bool kMask, class T, class F>
__device__ __forceinline__ void entries(const Row<T> &row, int thread, int lane, int lanes, F f)
{
    for (int i = thread + lane * kWideThreads; i < row.loose(); i += lanes * kWideThreads)
        f(row.template entry<kMask>(row.loose_at(i)), row.loose_at(i));
    for (int i = thread + lane * kWideThreads; i < row.packs; i += lanes * kWideThreads) {
        float v[Row<T>::kPack];
        row.template open<kMask>(row.raw(i), i, v);
#pragma unroll
        for (int k = 0; k < Row<T>::kPack; ++k)
            f(v[k], row.head + i * Row<T>::kPack + k);
    }
}

// A block a row: 2,047 rows of 65,536 16-bit entries, eight alternatives, 63 us,
// 4.3 TB/s, at 2.8 of 4 instructions a cycle; 20,000 of 2,000 39 us.
template <class T, int kWideThreads, bool kMask, bool kTop>
__global__ __launch_bounds__(kWideThreads) void logp_wide_kernel(const LogpArgs a, int top, float *logp, float *entropy,
                                                                 float *peak, float *logz, float *top_logp,
                                                                 int32_t *top_index)
{
    constexpr int kPack = Row<T>::kPack, kAhead = 4;
    __shared__ Scratch<kWideThreads> s;
    const int thread = threadIdx.x;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Row<T> row((const T *)a.logits + r * a.stride, kMask ? a.mask + r * a.mask_stride : nullptr, a.V);
        Sums q{kLowest, make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        int i = thread;
        for (; i + (kAhead - 1) * kWideThreads < row.packs; i += kAhead * kWideThreads) {
            uint4 raw[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                raw[k] = row.raw(i + k * kWideThreads);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                float v[kPack];
                row.template open<kMask>(raw[k], i + k * kWideThreads, v);
                take(q, v);
            }
        }
        for (; i < row.packs; i += kWideThreads) {
            float v[kPack];
            row.template open<kMask>(row.raw(i), i, v);
            take(q, v);
        }
        for (int j = thread; j < row.loose(); j += kWideThreads) {
            const float v[1] = {row.template entry<kMask>(row.loose_at(j))};
            take(q, v);
        }
        const float mine = q.m;
        const float m = reduce<kWideThreads>(mine, s.slots, [](float x, float y) { return fmaxf(x, y); });
        raise(q, m);
        auto plus = [](float x, float y) { return x + y; };
        const float e = reduce<kWideThreads>(q.e.x + q.e.y, s.slots, plus), ex = reduce<kWideThreads>(q.ex.x + q.ex.y, s.slots, plus);
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
        // (a thread without an entry stands for the lowest value, below which no entry is)
        const uint32_t highest = order_of(mine), floor = kth(highest, top, s);
        uint32_t again = __ballot_sync(~0u, highest >= floor);
        while (again) {  // the warp looks at one thread's entries after another
            const int lane = __ffs(again) - 1;
            again &= again - 1;
            entries<kWideThreads, kMask>(row, (thread & ~31) + lane, thread & 31, 32, [&](float v, int j) {
                const uint32_t u = order_of(v);
                if (u >= floor && u != 0) {
                    const int at = atomicAdd(&s.count, 1);
                    if (at < kListed)
                        s.list[at] = rank_key(v, j);
                }
            });
        }
        __syncthreads();
        const int count = s.count;
        if (count <= kListed && e == e) {
            for (int c = thread; c < count; c += kWideThreads) {
                const uint64_t key = s.list[c];
                int rank = 0;
                for (int o = 0; o < count; ++o)
                    rank += s.list[o] > key;
                if (rank < top) {
                    top_index[r * top + rank] = (int)~(uint32_t)key;
                    top_logp[r * top + rank] = (value_of((uint32_t)(key >> 32)) - m) - z;
                }
            }
            for (int k = count + thread; k < top; k += kWideThreads) {  // fewer than asked for
                top_index[r * top + k] = -1;
                top_logp[r * top + k] = no_value();
            }
        } else {
            uint64_t last = 0;
            for (int k = 0; k < top; ++k) {
                uint64_t best = 0;
                // (the first of all may have any key: of NaN at index 0 all bits are set)
                entries<kWideThreads, kMask>(row, thread, 0, 1, [&](float v, int j) {
                    const uint64_t key = rank_key(v, j);
                    best = (k == 0 || key < last) && key > best ? key : best;
                });
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    const uint64_t u = __shfl_xor_sync(~0u, best, o);
                    best = u > best ? u : best;
                }
                __syncthreads();
                if ((thread & 31) == 0)
                    s.best[thread >> 5] = best;
                __syncthreads();
                for (int w = 0; w < kWideThreads / 32; ++w)
                    best = s.best[w] > best ? s.best[w] : best;
                last = best;
                if (thread == 0) {
                    top_index[r * top + k] = best ? (int)~(uint32_t)best : -1;
                    top_logp[r * top + k] = best ? (value_of((uint32_t)(best >> 32)) - m) - z : no_value();
                }
            }
        }
        __syncthreads();  // (the list is the next row's)
    }
}

// A lane's entries of a row: kPer of them, kVec neighbours from each load.
template <class T, int kVec, int kLanes, int kPer>
struct Held {
    // the place of entry k
    __device__ static __forceinline__ int at(int k, int lane) { return (k / kVec * kLanes + lane) * kVec + k % kVec; }
    __device__ static __forceinline__ void load(float (&v)[kPer], const T *row, const uint8_t *mask, int V, int lane)
    {
#pragma unroll
        for (int c = 0; c < kPer; c += kVec) {
            const int j = at(c, lane);
            T q[kVec];
            if (j < V) {
                if constexpr (kVec == 1)
                    q[0] = row[j];
                else
                    *reinterpret_cast<uint4 *>(q) = *reinterpret_cast<const uint4 *>(row + j);
            }
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                v[c + e] = j < V && !(mask && mask[j + e] == 0) ? to_f32(q[e]) : no_value();
        }
    }
};

// kLanes lanes a row of at most kLanes kPer entries, all in registers: 65,536
// rows of 1,000 16-bit entries 39 us, with four alternatives 98; bound by issue.
template <class T, int kVec, int kLanes, int kPer, bool kTop>
__global__ __launch_bounds__(kNarrowThreads) void logp_narrow_kernel(const LogpArgs a, int top, float *logp,
                                                                     float *entropy, float *peak, float *logz,
                                                                     float *top_logp, int32_t *top_index)
{
    using H = Held<T, kVec, kLanes, kPer>;
    const int lane = threadIdx.x % kLanes;
    const int64_t r = ((int64_t)blockIdx.x * kNarrowThreads + threadIdx.x) / kLanes;
    const bool here = r < a.rows;  // (lanes without a row go along: shuffles are the warp's)
    const T *x = (const T *)a.logits + (here ? r : 0) * a.stride;
    const uint8_t *mask = a.mask ? a.mask + (here ? r : 0) * a.mask_stride : nullptr;
    const int64_t tok = here ? token_of(a.tokens, a.token_bytes, r) : -1;
    const bool given = tok >= 0 && tok < a.V;
    float v[kPer], m = kLowest;
    H::load(v, x, mask, a.V, lane);
    const float wanted = given && !(mask && mask[tok] == 0) ? to_f32(x[tok]) : no_value();
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        m = fmaxf(m, v[k]);
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1)
        m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    Sums q{m, make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
    for (int k = 0; k < kPer; k += 2)
        add(q, make_float2(v[k], v[k + 1]));
    float e = q.e.x + q.e.y, ex = q.ex.x + q.ex.y;
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1) {
        e += __shfl_xor_sync(~0u, e, o);
        ex += __shfl_xor_sync(~0u, ex, o);
    }
    const bool some = e != 0.0f;
    const float z = some ? logf(e) : no_value();
    if (here && lane == 0) {
        logp[r] = given ? (some ? (wanted - m) - z : no_value()) : 0.0f;
        if (entropy)
            entropy[r] = some ? z - ex / e : 0.0f;
        if (peak)
            peak[r] = some ? m : no_value();
        if (logz)
            logz[r] = z;
    }
    if (!kTop)
        return;
    auto put = [&](int i, uint32_t j, float value) {
        top_index[r * top + i] = (int)j;
        top_logp[r * top + i] = (value - m) - z;
    };
    auto put_none = [&](int i) {
        top_index[r * top + i] = -1;
        top_logp[r * top + i] = no_value();
    };
    if constexpr (kLanes < 32 && sizeof(T) == 2) {
        uint32_t u[kPer], best = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            u[k] = short_key<T>(v[k], H::at(k, lane));
            best = max(best, u[k]);
        }
        for (int i = 0; i < top; ++i) {
            uint32_t key = best;
#pragma unroll
            for (int o = kLanes / 2; o; o >>= 1)
                key = max(key, __shfl_xor_sync(~0u, key, o));
            if (here && lane == 0)
                key ? put(i, ~key & 0xffff, short_value<T>(key)) : put_none(i);
            if (key == best && key) {  // this lane's: the next of it
                best = 0;
#pragma unroll
                for (int k = 0; k < kPer; ++k)
                    best = max(best, u[k] < key ? u[k] : 0u);
            }
            __syncwarp();
        }
        return;
    }
    uint32_t u[kPer], best = 0;
    int at = 0;  // of this lane's largest
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        u[k] = order_of(v[k]);
        at = u[k] > best ? k : at;
        best = u[k] > best ? u[k] : best;
    }
    if (kLanes == 32 && top > 1) {
        __shared__ uint64_t lists[kNarrowThreads / 32][kShort];
        uint64_t *list = lists[threadIdx.x / 32];
        uint32_t left = best, floor = 0;
        for (int i = 0; i < top; ++i) {
            floor = __reduce_max_sync(~0u, left);
            const uint32_t holders = __ballot_sync(~0u, left == floor);
            if (lane == __ffs(holders) - 1)
                left = 0;
        }
        floor = max(floor, 1u);  // (0 is no entry)
        int mine = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            mine += u[k] >= floor;
        int to = mine;  // the end of this lane's on the list
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int before = __shfl_up_sync(~0u, to, o);
            to += lane >= o ? before : 0;
        }
        const int count = __shfl_sync(~0u, to, 31);
        if (count <= kShort) {
            to -= mine;
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (u[k] >= floor)
                    list[to++] = (uint64_t)u[k] << 32 | (uint32_t)~H::at(k, lane);
            __syncwarp();
            for (int c = lane; here && c < count; c += 32) {
                const uint64_t key = list[c];
                int rank = 0;
                for (int o = 0; o < count; ++o)
                    rank += list[o] > key;
                if (rank < top)
                    put(rank, ~(uint32_t)key, value_of((uint32_t)(key >> 32)));
            }
            for (int i = count + lane; here && i < top; i += 32)  // fewer than asked for
                put_none(i);
            return;
        }
    }
    for (int i = 0; i < top; ++i) {
        const uint64_t mine = best ? (uint64_t)best << 32 | (uint32_t)~H::at(at, lane) : 0;
        uint64_t key = mine;
#pragma unroll
        for (int o = kLanes / 2; o; o >>= 1) {
            const uint64_t other = __shfl_xor_sync(~0u, key, o);
            key = other > key ? other : key;
        }
        if (here && lane == 0)
            key ? put(i, ~(uint32_t)key, value_of((uint32_t)(key >> 32))) : put_none(i);
        if (key == mine && key) {  // this lane's: the next of it
            const int gone = at;
            best = 0;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                u[k] = k == gone ? 0 : u[k];
                at = u[k] > best ? k : at;
                best = u[k] > best ? u[k] : best;
            }
        }
        __syncwarp();
    }
}

// A thread a row of at most kMost entries, all in registers: a million rows of
// five 32-bit entries 12 us, with four alternatives 26.
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
    Sums q{m, make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
    const int64_t tok = token_of(a.tokens, a.token_bytes, r);
    float given = no_value();
#pragma unroll
    for (int j = 0; j < kMost; ++j)
        given = j == tok ? v[j] : given;
#pragma unroll
    for (int j = 0; j < kMost; j += 2)
        add(q, make_float2(v[j], v[j + 1]));
    const float e = q.e.x + q.e.y, ex = q.ex.x + q.ex.y;
    const bool some = e != 0.0f;
    const float z = some ? logf(e) : no_value();
    logp[r] = tok >= 0 && tok < a.V ? (some ? (given - m) - z : no_value()) : 0.0f;
    if (entropy)
        entropy[r] = some ? z - ex / e : 0.0f;
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

// What a row's gradient takes; c is dl + de entropy.
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
    s.c = s.dl + s.de * (dentropy ? entropy[r] : 0.0f);
    return s;
}

// exp2 with its smallest values: of 2^-126 and below the product with a log
// probability is not yet so small.
__device__ __forceinline__ float exp2_whole(float v)
{
    float r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Of an entry (-inf where it is masked), but for the token's own dlogp.
__device__ __forceinline__ float slope_at(const Slope &s, float x)
{
    const float lp = max_nan((x - s.m) - s.z, -200.0f);
    return -exp2_whole(lp * kLog2e) * fmaf(s.de, lp, s.c);
}

// An entry's gradient whole.
template <bool kMask>
__device__ __forceinline__ float gradient_at(const Slope &s, float x, int j)
{
    if (!s.some || (kMask && x == no_value()))
        return 0.0f;
    return slope_at(s, x) + (j == s.tok && x != no_value() ? s.dl : 0.0f);
}

// kLanes lanes a row of at most kLanes kPer entries: 65,536 rows of 1,000 16-bit
// ones 72 us, 3.7 TB/s.
template <class T, int kVec, int kLanes, int kPer>
__global__ __launch_bounds__(kNarrowThreads) void logp_narrow_grad_kernel(const LogpArgs a, const float *dlogp,
                                                                          const float *dentropy, const float *peak,
                                                                          const float *logz, const float *entropy,
                                                                          T *dlogits, int64_t dstride)
{
    using H = Held<T, kVec, kLanes, kPer>;
    const int lane = threadIdx.x % kLanes;
    const int64_t r = ((int64_t)blockIdx.x * kNarrowThreads + threadIdx.x) / kLanes;
    if (r >= a.rows)
        return;
    float v[kPer];
    H::load(v, (const T *)a.logits + r * a.stride, a.mask ? a.mask + r * a.mask_stride : nullptr, a.V, lane);
    const Slope s = slope_of(a, r, dlogp, dentropy, peak, logz, entropy);
    T *dx = dlogits + r * dstride;
#pragma unroll
    for (int c = 0; c < kPer; c += kVec) {
        const int j = H::at(c, lane);
        if (j >= a.V)
            continue;
        T o[kVec];
        // (an absent entry's logit is -inf and its gradient 0 with or without a mask)
#pragma unroll
        for (int e = 0; e < kVec; ++e)
            o[e] = from_f32<T>(gradient_at<true>(s, v[c + e], j + e));
        if constexpr (kVec == 1)
            dx[j] = o[0];
        else
            *reinterpret_cast<uint4 *>(dx + j) = *reinterpret_cast<const uint4 *>(o);
    }
}

// A block takes a part of a row, or a warp a row: 2,047 rows of 65,536 16-bit
// entries 96 us, 5.6 TB/s; 20,000 of 2,000, by warps, 36 us, 4.4 TB/s.
template <class T, int kLanes, bool kMask>
__global__ __launch_bounds__(kGradThreads) void logp_wide_grad_kernel(const LogpArgs a, const float *dlogp,
                                                                      const float *dentropy, const float *peak,
                                                                      const float *logz, const float *entropy,
                                                                      T *dlogits, int64_t dstride, bool packed)
{
    constexpr int kPack = Row<T>::kPack, kAhead = 4;
    const int64_t r = (int64_t)blockIdx.x * (kGradThreads / kLanes) + threadIdx.x / kLanes;
    if (r >= a.rows)
        return;
    const Row<T> row((const T *)a.logits + r * a.stride, kMask ? a.mask + r * a.mask_stride : nullptr, a.V);
    const Slope s = slope_of(a, r, dlogp, dentropy, peak, logz, entropy);
    T *dx = dlogits + r * dstride;
    const int thread = threadIdx.x % kLanes + blockIdx.y * kLanes, step = kLanes * gridDim.y;
    if (!packed) {  // dlogits' rows begin elsewhere in 16 bytes than those of logits
        for (uint32_t j = thread; j < (uint32_t)a.V; j += step)  // (the last step may go beyond an int)
            dx[j] = from_f32<T>(gradient_at<kMask>(s, row.template entry<kMask>(j), j));
        return;
    }
    for (int i = thread; i < row.loose(); i += step) {
        const int j = row.loose_at(i);
        dx[j] = from_f32<T>(gradient_at<kMask>(s, row.template entry<kMask>(j), j));
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
                    o[e] = from_f32<T>(gradient_at<kMask>(s, v[e], j + e));
            }
            *reinterpret_cast<uint4 *>(dx + j) = out;
        }
    }
}

// A thread a row.  The block's rows of 12 bytes or more, where they lie side by
// side (kSide), go through shared memory, which lets neighbouring threads touch
// neighbouring places: a million rows of seven 32-bit entries 21 us, straight 33,
// of five 17 and 21, of seven 16-bit ones 18.5 and 25; of five, of ten bytes,
// straight is the faster by a tenth, 16.5.
template <class T, bool kMask, bool kSide>
__global__ __launch_bounds__(kTinyThreads) void logp_grad_tiny_kernel(const LogpArgs a, const float *dlogp,
                                                                      const float *dentropy, const float *peak,
                                                                      const float *logz, const float *entropy,
                                                                      T *dlogits, int64_t dstride)
{
    __shared__ T rows[kSide ? kTinyThreads * kTiny : 1];
    __shared__ uint8_t there[kSide && kMask ? kTinyThreads * kTiny : 1];
    const int64_t r0 = (int64_t)blockIdx.x * kTinyThreads, r = r0 + threadIdx.x;
    const int count = kSide ? (int)(a.rows - r0 < kTinyThreads ? a.rows - r0 : kTinyThreads) * a.V : 0;
    const T *from = (const T *)a.logits + r0 * a.V;
    T *to = dlogits + r0 * a.V;
    if (kSide) {
#pragma unroll
        for (int k = 0; k < kTiny; ++k) {
            const int i = k * kTinyThreads + threadIdx.x;
            if (i < count) {
                rows[i] = from[i];
                if (kMask)
                    there[i] = a.mask[r0 * a.V + i];
            }
        }
        __syncthreads();
    }
    if (r < a.rows) {
        const T *x = kSide ? rows + threadIdx.x * a.V : (const T *)a.logits + r * a.stride;
        const uint8_t *mask = !kMask ? nullptr : kSide ? there + threadIdx.x * a.V : a.mask + r * a.mask_stride;
        T *dx = kSide ? rows + threadIdx.x * a.V : dlogits + r * dstride;
        const Slope s = slope_of(a, r, dlogp, dentropy, peak, logz, entropy);
#pragma unroll 8
        for (int j = 0; j < a.V; ++j) {
            const float v = kMask && mask[j] == 0 ? no_value() : to_f32(x[j]);
            dx[j] = from_f32<T>(gradient_at<kMask>(s, v, j));
        }
    }
    if (kSide) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kTiny; ++k) {
            const int i = k * kTinyThreads + threadIdx.x;
            if (i < count)
                to[i] = rows[i];
        }
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

// Calls f with the lanes and the entries a lane for rows of V entries.
template <class F>
void with_lanes(int V, F f)
{
    using std::integral_constant;
    const integral_constant<int, 16> sixteen;
    if (V <= 32)
        f(integral_constant<int, 2>(), sixteen);
    else if (V <= 64)
        f(integral_constant<int, 4>(), sixteen);
    else if (V <= 128)
        f(integral_constant<int, 8>(), sixteen);
    else if (V <= 256)
        f(integral_constant<int, 16>(), sixteen);
    else if (V <= 512)
        f(integral_constant<int, 32>(), sixteen);
    else
        f(integral_constant<int, 32>(), integral_constant<int, 32>());
}

// Whether rows take a block of 128 threads (else one of 512): many of them, of
// up to 32 KB.  Of 16-bit entries, small block and large: 4,864 rows of 2,000 11
// and 24 us, of 16,384 34 and 44, with four alternatives 50 and 62; 608 of 2,000
// 4.6 and 6.5, of 8,192 6.7 and 8.5; but 304 of 8,192 with alternatives 10.8 and
// 8.5, 608 of 12,000 13.1 and 11.9, 2,432 of 24,000 44 and 40.
bool small_blocks(int64_t rows, int64_t bytes) { return bytes <= 32768 && rows >= (bytes <= 16384 ? 608 : 1216); }

// Whether a row's gradient takes a warp (else blocks, of 16,384 entries each):
// 4,864 rows of 4,096 16-bit entries take 17 us by warps and 31 by blocks, 2,432
// of 8,192 18.5 and 20.7, of 2,000 32-bit ones 10.3 and 12.4; but 304 of 8,192
// 12.4 and 6.2, 2,432 of 8,192 32-bit ones 33 and 29; 608 of 1,500 6.2 either way.
bool by_warps(int64_t rows, int64_t bytes) { return bytes <= 16384 && rows >= 1216; }

// Rows of whole 16-byte packs.
bool packs(const void *p, int64_t rows, int V, int64_t stride, int64_t e)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && V * e % 16 == 0 && (rows <= 1 || stride * e % 16 == 0);
}

}  // namespace

cudaError_t launch_logp(const LogpArgs &a, int top, float *logp, float *entropy, float *peak, float *logz,
                        float *top_logp, int32_t *top_index, cudaStream_t st)
{
    with_type(a.dtype, [&](auto v) {
        using T = decltype(v);
        if (a.V > kTiny && a.V <= kNarrow) {
            with_lanes(a.V, [&](auto lanes, auto per) {
                auto run = [&](auto kernel) {
                    kernel<<<(unsigned)up(a.rows * lanes.value, kNarrowThreads), kNarrowThreads, 0, st>>>(
                        a, top, logp, entropy, peak, logz, top_logp, top_index);
                };
                with_flag(top > 0, [&](auto tops) {
                    if (packs(a.logits, a.rows, a.V, a.stride, sizeof(T)))
                        run(logp_narrow_kernel<T, 16 / sizeof(T), lanes.value, per.value, tops.value>);
                    else
                        run(logp_narrow_kernel<T, 1, lanes.value, per.value, tops.value>);
                });
            });
            return;
        }
        with_flag(a.mask != nullptr, [&](auto mask) {
            if (a.V <= kTiny) {
                logp_tiny_kernel<T, kTiny, mask.value><<<(unsigned)up(a.rows, kTinyThreads), kTinyThreads, 0, st>>>(
                    a, top, logp, entropy, peak, logz, top_logp, top_index);
                return;
            }
            with_flag(top > 0, [&](auto tops) {
                auto run = [&](auto kernel, int threads) {
                    const int64_t most = 152 * 4 * (2048 / threads);
                    kernel<<<(unsigned)(a.rows < most ? a.rows : most), threads, 0, st>>>(a, top, logp, entropy, peak,
                                                                                         logz, top_logp, top_index);
                };
                if (small_blocks(a.rows, a.V * (int64_t)sizeof(T)))
                    run(logp_wide_kernel<T, 128, mask.value, tops.value>, 128);
                else
                    run(logp_wide_kernel<T, 512, mask.value, tops.value>, 512);
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
        const bool whole = packs(a.logits, a.rows, a.V, a.stride, e) && packs(dlogits, a.rows, a.V, dlogit_stride, e);
        // (two lanes for eight 32-bit entries: 44 us for 2 M rows, a thread for them 72; of 16 bits 52 and 50)
        if (a.V <= kNarrow && (a.V > kTiny || (whole && a.V * e >= 32))) {
            with_lanes(a.V, [&](auto lanes, auto per) {
                auto run = [&](auto kernel) {
                    kernel<<<(unsigned)up(a.rows * lanes.value, kNarrowThreads), kNarrowThreads, 0, st>>>(
                        a, dlogp, dentropy, peak, logz, entropy, dx, dlogit_stride);
                };
                if (whole)
                    run(logp_narrow_grad_kernel<T, 16 / sizeof(T), lanes.value, per.value>);
                else
                    run(logp_narrow_grad_kernel<T, 1, lanes.value, per.value>);
            });
            return;
        }
        // whether dlogits' rows begin where in 16 bytes those of logits do
        const bool packed = ((reinterpret_cast<uintptr_t>(dlogits) ^ reinterpret_cast<uintptr_t>(a.logits)) & 15) == 0 &&
                            (a.rows <= 1 || (dlogit_stride - a.stride) * e % 16 == 0);
        with_flag(a.mask != nullptr, [&](auto mask) {
            if (a.V <= kTiny) {
                const bool side = a.V * e >= 12 && a.stride == a.V && dlogit_stride == a.V &&
                                  (!mask.value || a.mask_stride == a.V);
                with_flag(side, [&](auto by_side) {
                    logp_grad_tiny_kernel<T, mask.value, by_side.value>
                        <<<(unsigned)up(a.rows, kTinyThreads), kTinyThreads, 0, st>>>(a, dlogp, dentropy, peak, logz,
                                                                                      entropy, dx, dlogit_stride);
                });
            } else if (by_warps(a.rows, a.V * e)) {
                logp_wide_grad_kernel<T, 32, mask.value>
                    <<<(unsigned)up(a.rows, kGradThreads / 32), kGradThreads, 0, st>>>(
                        a, dlogp, dentropy, peak, logz, entropy, dx, dlogit_stride, packed);
            } else {
                const int parts = (int)up(a.V, 16384);  // (of a row; blocks of some 16,384 entries)
                logp_wide_grad_kernel<T, kGradThreads, mask.value>
                    <<<dim3((unsigned)a.rows, (unsigned)(parts < 65535 ? parts : 65535)), kGradThreads, 0, st>>>(
                        a, dlogp, dentropy, peak, logz, entropy, dx, dlogit_stride, packed);
            }
        });
    });
    return cudaGetLastError();
}

}  // namespace av
