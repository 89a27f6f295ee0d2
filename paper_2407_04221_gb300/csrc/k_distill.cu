// k_distill.cu -- how far the distribution over a row of logits is from a
// teacher's over its few alternatives, and the gradient.  With temperature h,
// m the row's largest logit, and over the teacher's entries t_i of index j_i
// that are there:
//   logz = log sum exp((x - m) / h),  log p_j = (x_j - m) / h - logz
//   q = softmax(t / h),  kl = sum q_i (log q_i - log p_{j_i})
//   dx_j = dkl / h (p_j - sum of q_i over j_i = j)
//
// Both passes read the logits once and are bound by memory.  Rows of up to eight
// entries take a thread, of up to 1,024 a group of lanes that holds them in
// registers, longer ones a block, or parts of one.  The teacher's entries are
// some tens: a warp weighs them beside the row.  Backward, the row is written as
// if there were no teacher and the entries that it names are written again after,
// by the same block, each by the first of the alternatives that name it.
//
// Addition has one order throughout: equal rows give equal bits.
#include "rows.cuh"

namespace av {
namespace {

constexpr int kTiny = 8;           // entries of a row that a thread takes
constexpr int kTinyThreads = 128;
constexpr int kNarrow = 1024;      // entries of a row that a group of lanes takes
constexpr int kNarrowThreads = 256;
constexpr int kGradThreads = 256;

// ------------------------------------------------------------ the teacher

__device__ __forceinline__ float teacher_of(const void *p, int dtype, int64_t i)
{
    return dtype == AV_F32 ? ((const float *)p)[i]
                           : dtype == AV_BF16 ? to_f32(((const __nv_bfloat16 *)p)[i]) : to_f32(((const __half *)p)[i]);
}

// Entry i of row r: its index in the row, or -1 where it is not there.
__device__ __forceinline__ int taught(const DistillArgs &a, int64_t r, int i, float &t)
{
    const int64_t at = r * a.k + i, j = a.index_bytes == 4 ? ((const int32_t *)a.index)[at] : ((const int64_t *)a.index)[at];
    t = no_value();
    if (j < 0 || j >= a.V)
        return -1;
    t = teacher_of(a.teacher, a.teacher_dtype, at);
    return t == no_value() ? -1 : (int)j;
}

template <int kLanes>
__device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1)
        v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1)
        v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// The divergence of a row, by kLanes lanes of a whole warp; x: its logits (-inf
// where absent), m and z its peak and log sum.  sum q (log q - log p) with e_i the
// teacher's exponentials below its peak and s their sum:
//   (sum e_i ((t_i - top) / h - (x_i - m) / h)) / s - log s + logz
// `j0`, `t0`: this lane's first alternative, where it has been read ahead (65,536 rows of 1,000 take 52 us without, 57 so).
template <int kLanes, bool kAhead, class F>
__device__ __forceinline__ float divergence(const DistillArgs &a, int64_t r, bool here, int lane, int j0, float t0, float m, float z, F x)
{
    float top = t0;
    int some = j0 >= 0;
    const int from = kAhead ? lane + kLanes : lane;
    for (int i = from; here && i < a.k; i += kLanes) {
        float t;
        some |= taught(a, r, i, t) >= 0;
        top = fmaxf(top, t);
    }
    top = lanes_max<kLanes>(top);
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1)
        some |= __shfl_xor_sync(~0u, some, o);
    float sum = 0.0f, mix = 0.0f;
    auto weigh_in = [&](int j, float t) {
        if (j < 0)
            return;
        const float d = (t - top) * a.inv, e = exp2_whole(d * kLog2e);
        sum += e;
        if (e != 0.0f)  // (an alternative of no weight, below 2^-149, may be one that the student does not have)
            mix += e * (d - (x(j) - m) * a.inv);
    };
    if (kAhead)
        weigh_in(j0, t0);
    for (int i = from; here && i < a.k; i += kLanes) {
        float t;
        const int j = taught(a, r, i, t);
        weigh_in(j, t);
    }
    sum = lanes_sum<kLanes>(sum);
    mix = lanes_sum<kLanes>(mix);
    if (!some)
        return 0.0f;
    if (z == no_value())  // nothing is left of the student's row
        return sum == sum ? INFINITY : sum;
    return mix / sum - logf(sum) + z;
}

// ------------------------------------------------------------ forward

// The running maximum and the sum of exp((x - m) / h), c = log2(e) / h.
struct Total {
    float m;
    float2 e;
};
__device__ __forceinline__ void raise(Total &s, float m, float c)
{
    const float k = exp2_fast((s.m - m) * c);
    s.e = mul2(s.e, make_float2(k, k));
    s.m = m;
}
template <int kN>
__device__ __forceinline__ void take(Total &s, const float (&x)[kN], float c)
{
    float m = x[0];
#pragma unroll
    for (int k = 1; k < kN; ++k)
        m = fmaxf(m, x[k]);
    if (m > s.m)
        raise(s, m, c);
    const float2 low = make_float2(-s.m, -s.m), c2 = make_float2(c, c);
#pragma unroll
    for (int k = 0; k < kN; k += 2) {
        const float2 t = mul2(add2(make_float2(x[k], k + 1 < kN ? x[k + 1] : no_value()), low), c2);
        s.e = add2(s.e, make_float2(exp2_fast(t.x), exp2_fast(t.y)));
    }
}

__device__ __forceinline__ void leave(const DistillOut &o, int64_t r, float kl, float m, float z)
{
    o.kl[r] = kl;
    if (o.peak)
        o.peak[r] = z == no_value() || (z != z && m != INFINITY) ? z : m;  // (NaN has not been compared)
    if (o.logz)
        o.logz[r] = z;
}

// A block a row: 4,096 rows of 65,536 16-bit entries 85 us, 6.3 TB/s; 3,001 of 10,007 32-bit ones, whose rows start on any 4
// bytes, 24, 5.0 TB/s.
template <class T, int kWideThreads, bool kMask>
__global__ __launch_bounds__(kWideThreads) void distill_wide_kernel(const DistillArgs a, const DistillOut o)
{
    constexpr int kPack = Row<T>::kPack, kAhead = 4;
    __shared__ float slots[kWideThreads / 32];
    const int thread = threadIdx.x;
    const float c = a.inv * kLog2e;
    const int64_t r = blockIdx.x;
    float t0 = no_value();
    const int j0 = thread < min(a.k, 32) ? taught(a, r, thread, t0) : -1;
    const Row<T> row((const T *)a.logits + r * a.stride, kMask ? a.mask + r * a.mask_stride : nullptr, a.V);
    Total q{kLowest, make_float2(0.0f, 0.0f)};
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
            take(q, v, c);
        }
    }
    for (; i < row.packs; i += kWideThreads) {
        float v[kPack];
        row.template open<kMask>(row.raw(i), i, v);
        take(q, v, c);
    }
    for (int j = thread; j < row.loose(); j += kWideThreads) {
        const float v[1] = {row.template entry<kMask>(row.loose_at(j))};
        take(q, v, c);
    }
    const float m = reduce<kWideThreads>(q.m, slots, [](float x, float y) { return fmaxf(x, y); });
    raise(q, m, c);
    const float e = reduce<kWideThreads>(q.e.x + q.e.y, slots, [](float x, float y) { return x + y; });
    const float z = e != 0.0f ? logf(e) : no_value();  // (NaN counts)
    if (thread < 32) {
        const float kl = divergence<32, true>(a, r, true, thread, j0, t0, m, z, [&](int j) { return row.template entry<kMask>(j); });
        if (thread == 0)
            leave(o, r, kl, m, z);
    }
}

// kLanes lanes a row of at most kLanes kPer entries: 65,536 rows of 1,000 16-bit ones with 32 alternatives 52 us, bound by
// issue, a quarter of it the teacher's.
template <class T, int kVec, int kLanes, int kPer>
__global__ __launch_bounds__(kNarrowThreads) void distill_narrow_kernel(const DistillArgs a, const DistillOut o)
{
    using H = Held<T, kVec, kLanes, kPer>;
    const int lane = threadIdx.x % kLanes;
    const int64_t r = ((int64_t)blockIdx.x * kNarrowThreads + threadIdx.x) / kLanes;
    const bool here = r < a.rows;  // (lanes without a row go along: shuffles are the warp's)
    const T *x = (const T *)a.logits + (here ? r : 0) * a.stride;
    const uint8_t *mask = a.mask ? a.mask + (here ? r : 0) * a.mask_stride : nullptr;
    float v[kPer], m = kLowest;
    H::load(v, x, mask, a.V, lane);
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        m = fmaxf(m, v[k]);
    Total q{lanes_max<kLanes>(m), make_float2(0.0f, 0.0f)};
    take(q, v, a.inv * kLog2e);
    const float e = lanes_sum<kLanes>(q.e.x + q.e.y), z = e != 0.0f ? logf(e) : no_value();
    const float kl = divergence<kLanes, false>(a, r, here, lane, -1, no_value(), q.m, z,
                                        [&](int j) { return mask && mask[j] == 0 ? no_value() : to_f32(x[j]); });
    if (here && lane == 0)
        leave(o, r, kl, q.m, z);
}

// All of a row's alternatives, at most kTiny, by one thread; -1 where one is not there.
template <class I>
__device__ __forceinline__ void taught_all(const DistillArgs &a, int64_t r, int (&at)[kTiny], float (&t)[kTiny])
{
    const I *index = (const I *)a.index + r * a.k;
    I j[kTiny];
#pragma unroll
    for (int i = 0; i < kTiny; ++i)
        j[i] = i < a.k ? index[i] : -1;
    if (a.teacher_dtype == AV_F32) {
        const float *teacher = (const float *)a.teacher + r * a.k;
#pragma unroll
        for (int i = 0; i < kTiny; ++i)
            t[i] = i < a.k ? teacher[i] : no_value();
    } else {
#pragma unroll
        for (int i = 0; i < kTiny; ++i)
            t[i] = i < a.k ? teacher_of(a.teacher, a.teacher_dtype, r * a.k + i) : no_value();
    }
#pragma unroll
    for (int i = 0; i < kTiny; ++i) {
        const bool there = j[i] >= 0 && j[i] < a.V && t[i] != no_value();
        at[i] = there ? (int)j[i] : -1;
        t[i] = there ? t[i] : no_value();
    }
}
__device__ __forceinline__ void taught_all(const DistillArgs &a, int64_t r, int (&at)[kTiny], float (&t)[kTiny])
{
    if (a.index_bytes == 4)
        taught_all<int32_t>(a, r, at, t);
    else
        taught_all<int64_t>(a, r, at, t);
}

// A thread a row: 262,144 of five 32-bit entries 9 us, and 9 back; bound by issue.  (Rows by way of shared memory, in whole
// lines, took 15 and 12.6 where these took 12.8 and 10.4.)
template <class T, bool kMask>
__global__ __launch_bounds__(kTinyThreads) void distill_tiny_kernel(const DistillArgs a, const DistillOut o)
{
    const int64_t r = (int64_t)blockIdx.x * kTinyThreads + threadIdx.x;
    if (r >= a.rows)
        return;
    const T *x = (const T *)a.logits + r * a.stride;
    const uint8_t *mask = kMask ? a.mask + r * a.mask_stride : nullptr;
    int at[kTiny];
    float t[kTiny], v[kTiny], m = kLowest;
    taught_all(a, r, at, t);
#pragma unroll
    for (int j = 0; j < kTiny; ++j) {
        v[j] = j < a.V && (!kMask || mask[j] != 0) ? to_f32(x[j]) : no_value();
        m = fmaxf(m, v[j]);
    }
    Total q{m, make_float2(0.0f, 0.0f)};
    take(q, v, a.inv * kLog2e);
    const float e = q.e.x + q.e.y, z = e != 0.0f ? logf(e) : no_value();
    float top = no_value(), sum = 0.0f, mix = 0.0f, kl = 0.0f;
    bool some = false;
#pragma unroll
    for (int i = 0; i < kTiny; ++i) {
        some |= at[i] >= 0;
        top = fmaxf(top, t[i]);
    }
#pragma unroll
    for (int i = 0; i < kTiny; ++i) {
        if (i >= a.k)
            break;
        if (at[i] < 0)
            continue;
        const float d = (t[i] - top) * a.inv, w = exp2_whole(d * kLog2e);
        sum += w;
        if (w != 0.0f) {
            const float low = kMask && mask[at[i]] == 0 ? no_value() : to_f32(x[at[i]]);
            mix += w * (d - (low - m) * a.inv);
        }
    }
    if (some)
        kl = z == no_value() ? (sum == sum ? INFINITY : sum) : mix / sum - logf(sum) + z;
    leave(o, r, kl, m, z);
}

// ------------------------------------------------------------ backward

// What a row's gradient takes: p = exp2((x - m) c - zc), times up; nothing where it is not live.
struct Slope {
    float m, c, zc, up;
    bool live, plain;  // plain: an entry of -inf makes a gradient of 0
};
__device__ __forceinline__ Slope slope_of(const DistillArgs &a, int64_t r, const float *dkl, const float *peak, const float *logz)
{
    const float z = logz[r], up = dkl[r] * a.inv;
    return {peak[r], a.inv * kLog2e, z * kLog2e, up, z != no_value(), fabsf(up) <= 3.402823466e38f && fabsf(z) <= 3.402823466e38f};
}
__device__ __forceinline__ float share(const Slope &s, float x) { return exp2_whole(fmaf(x - s.m, s.c, -s.zc)); }

// An entry without the teacher's part; 0 where it is absent.
__device__ __forceinline__ float gradient_at(const Slope &s, float x)
{
    return s.live && x != no_value() ? share(s, x) * s.up : 0.0f;
}

// kN entries, of a row that is live and plain or not.
template <class T, int kN>
__device__ __forceinline__ void gradients(const Slope &s, const float (&x)[kN], T *o)
{
    if (s.live && s.plain) {
        const float2 low = make_float2(-s.m, -s.m), c = make_float2(s.c, s.c), zc = make_float2(-s.zc, -s.zc),
                     up = make_float2(s.up, s.up);
#pragma unroll
        for (int e = 0; e < kN; e += 2) {
            const float2 t = fma2(add2(make_float2(x[e], x[e + 1]), low), c, zc);
            const float2 g = mul2(make_float2(exp2_whole(t.x), exp2_whole(t.y)), up);
            o[e] = from_f32<T>(g.x);
            o[e + 1] = from_f32<T>(g.y);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
            o[e] = from_f32<T>(gradient_at(s, x[e]));
    }
}

// The teacher's weights into `weight`, `at`, by kLanes lanes of a whole warp; whether there is one.
template <int kLanes>
__device__ __forceinline__ bool weigh(const DistillArgs &a, int64_t r, bool here, int lane, int *at, float *weight)
{
    float top = no_value();
    int some = 0;
    for (int i = lane; here && i < a.k; i += kLanes) {
        float t;
        at[i] = taught(a, r, i, t);
        some |= at[i] >= 0;
        weight[i] = t;
        top = fmaxf(top, t);
    }
    top = lanes_max<kLanes>(top);
    float sum = 0.0f;
    for (int i = lane; here && i < a.k; i += kLanes) {
        const float e = at[i] >= 0 ? exp2_whole((weight[i] - top) * a.inv * kLog2e) : 0.0f;
        weight[i] = e;
        sum += e;
    }
    sum = lanes_sum<kLanes>(sum);
    const float part = 1.0f / sum;
    for (int i = lane; here && i < a.k; i += kLanes)
        weight[i] *= part;
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1)
        some |= __shfl_xor_sync(~0u, some, o);
    __syncwarp();
    return some != 0;
}

constexpr int kSeen = 256;  // words of bits for the entries that have been named

// Whether two alternatives name the same entry, or may: long rows' share a bit with others.  By kLanes lanes of a whole
// warp; `seen`: a word for 32 entries, or kSeen.
template <int kLanes>
__device__ __forceinline__ bool named_twice(const DistillArgs &a, bool here, int lane, const int *at, uint32_t *seen)
{
    const int words = a.V <= kSeen * 32 ? (a.V + 31) / 32 : kSeen;
    for (int i = lane; i < words; i += kLanes)
        seen[i] = 0;
    __syncwarp();
    int again = 0;
    for (int i = lane; here && i < a.k; i += kLanes)
        if (at[i] >= 0) {
            const uint32_t bit = 1u << (at[i] & 31);
            again |= (atomicOr(&seen[at[i] >> 5 & (kSeen - 1)], bit) & bit) != 0;
        }
#pragma unroll
    for (int o = kLanes / 2; o; o >>= 1)
        again |= __shfl_xor_sync(~0u, again, o);
    return again != 0;
}

// The entries that the teacher names, written again: those from lo up to hi.  Where none is named twice each alternative
// is its entry's only one.
template <class T, class F>
__device__ __forceinline__ void write_named(const Slope &s, int k, bool twice, const int *at, const float *weight, int first, int step,
                                            int64_t lo, int64_t hi, T *dx, F x)
{
    for (int i = first; i < k; i += step) {
        const int j = at[i];
        if (j < lo || j >= hi || j < 0)
            continue;
        float w = twice ? 0.0f : weight[i];
        bool mine = true;  // the first of those that name it
        for (int o = 0; twice && o < k; ++o)
            if (at[o] == j) {
                mine &= o >= i;
                w += weight[o];
            }
        const float v = x(j);
        if (mine && v != no_value() && s.live)
            dx[j] = from_f32<T>((share(s, v) - w) * s.up);
    }
}

// kLanes lanes a row of at most kLanes kPer entries: 65,536 rows of 1,000 16-bit ones 78 us, 3.4 TB/s.
template <class T, int kVec, int kLanes, int kPer>
__global__ __launch_bounds__(kNarrowThreads) void distill_narrow_grad_kernel(const DistillArgs a, const float *dkl,
                                                                             const float *peak, const float *logz,
                                                                             T *dlogits, int64_t dstride)
{
    using H = Held<T, kVec, kLanes, kPer>;
    extern __shared__ float scratch[];  // [rows of the block][k] weights, the same of indices
    const int lane = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
    float *weight = scratch + slot * a.k;
    int *at = reinterpret_cast<int *>(scratch + kNarrowThreads / kLanes * a.k) + slot * a.k;
    __shared__ uint32_t seen_bits[kNarrowThreads / kLanes][kLanes * kPer / 32];
    const int64_t r = (int64_t)blockIdx.x * (kNarrowThreads / kLanes) + slot;
    const bool here = r < a.rows;
    const T *x = (const T *)a.logits + (here ? r : 0) * a.stride;
    const uint8_t *mask = a.mask ? a.mask + (here ? r : 0) * a.mask_stride : nullptr;
    float v[kPer];
    H::load(v, x, mask, a.V, lane);
    Slope s = slope_of(a, here ? r : 0, dkl, peak, logz);
    s.live &= weigh<kLanes>(a, r, here, lane, at, weight);
    const bool twice = named_twice<kLanes>(a, here, lane, at, seen_bits[slot]);
    T *dx = dlogits + r * dstride;
    if (here) {
        alignas(16) T o[kPer];
        gradients<T>(s, v, o);
#pragma unroll
        for (int c = 0; c < kPer; c += kVec) {
            const int j = H::at(c, lane);
            if (j >= a.V)
                continue;
            if constexpr (kVec == 1)
                dx[j] = o[c];
            else
                *reinterpret_cast<uint4 *>(dx + j) = *reinterpret_cast<const uint4 *>(o + c);
        }
    }
    __syncwarp();
    if (here)
        write_named(s, a.k, twice, at, weight, lane, kLanes, 0, a.V, dx,
                    [&](int j) { return mask && mask[j] == 0 ? no_value() : to_f32(x[j]); });
}

// A block takes a part of a row, or a warp a row: 4,096 rows of 65,536 16-bit entries 167 us, 6.4 TB/s; 3,001 of 10,007
// 32-bit ones 47, 5.1 TB/s.
template <class T, int kLanes, bool kMask>
__global__ __launch_bounds__(kGradThreads) void distill_wide_grad_kernel(const DistillArgs a, const float *dkl,
                                                                         const float *peak, const float *logz, T *dlogits,
                                                                         int64_t dstride, bool packed)
{
    constexpr int kPack = Row<T>::kPack, kAhead = 4, kSlots = kGradThreads / kLanes;
    extern __shared__ float scratch[];
    __shared__ uint32_t seen_bits[kSlots][kSeen];
    __shared__ int flags;
    const int slot = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    float *weight = scratch + slot * a.k;
    int *at = reinterpret_cast<int *>(scratch + kSlots * a.k) + slot * a.k;
    uint32_t *seen = seen_bits[slot];
    const int64_t r = (int64_t)blockIdx.x * kSlots + slot;
    if (r >= a.rows)  // (whole warps)
        return;
    const Row<T> row((const T *)a.logits + r * a.stride, kMask ? a.mask + r * a.mask_stride : nullptr, a.V);
    Slope s = slope_of(a, r, dkl, peak, logz);
    bool twice;
    if constexpr (kLanes == 32) {
        s.live &= weigh<32>(a, r, true, lane, at, weight);
        twice = named_twice<32>(a, true, lane, at, seen);
    } else {
        if (threadIdx.x < 32) {
            const bool any = weigh<32>(a, r, true, lane, at, weight), again = named_twice<32>(a, true, lane, at, seen);
            if (lane == 0)
                flags = (any ? 1 : 0) | (again ? 2 : 0);
        }
        __syncthreads();
        s.live &= (flags & 1) != 0;
        twice = (flags & 2) != 0;
    }
    T *dx = dlogits + r * dstride;
    // this block's part: packs from p0 to p1, entries from j0 to j1
    const int parts = (int)gridDim.y, part = (int)blockIdx.y;
    int64_t j0 = (int64_t)a.V * part / parts, j1 = (int64_t)a.V * (part + 1) / parts;
    if (!packed) {  // dlogits' rows begin elsewhere in 16 bytes than those of logits
        for (int64_t j = j0 + lane; j < j1; j += kLanes)
            dx[j] = from_f32<T>(gradient_at(s, row.template entry<kMask>((int)j)));
    } else {
        const int p0 = (int)((int64_t)row.packs * part / parts), p1 = (int)((int64_t)row.packs * (part + 1) / parts);
        const int tail = row.head + row.packs * kPack;
        j0 = part == 0 ? 0 : row.head + (int64_t)p0 * kPack;
        j1 = part == parts - 1 ? a.V : row.head + (int64_t)p1 * kPack;
        if (part == 0)
            for (int j = lane; j < row.head; j += kLanes)
                dx[j] = from_f32<T>(gradient_at(s, row.template entry<kMask>(j)));
        if (part == parts - 1)
            for (int64_t j = tail + lane; j < a.V; j += kLanes)
                dx[j] = from_f32<T>(gradient_at(s, row.template entry<kMask>((int)j)));
        for (int i0 = p0 + lane; i0 < p1; i0 += kAhead * kLanes) {
            uint4 raw[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                raw[k] = i0 + k * kLanes < p1 ? row.raw(i0 + k * kLanes) : uint4{};
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int i = i0 + k * kLanes;
                if (i >= p1)
                    break;
                float v[kPack];
                row.template open<kMask>(raw[k], i, v);
                uint4 out;
                gradients<T>(s, v, reinterpret_cast<T *>(&out));
                *reinterpret_cast<uint4 *>(dx + row.head + (int64_t)i * kPack) = out;
            }
        }
    }
    if constexpr (kLanes == 32)
        __syncwarp();
    else
        __syncthreads();
    write_named(s, a.k, twice, at, weight, lane, kLanes, j0, j1, dx, [&](int j) { return row.template entry<kMask>(j); });
}

template <class T, bool kMask>
__global__ __launch_bounds__(kTinyThreads) void distill_tiny_grad_kernel(const DistillArgs a, const float *dkl,
                                                                         const float *peak, const float *logz, T *dlogits,
                                                                         int64_t dstride)
{
    const int64_t r = (int64_t)blockIdx.x * kTinyThreads + threadIdx.x;
    if (r >= a.rows)
        return;
    const T *x = (const T *)a.logits + r * a.stride;
    const uint8_t *mask = kMask ? a.mask + r * a.mask_stride : nullptr;
    Slope s = slope_of(a, r, dkl, peak, logz);
    int at[kTiny];
    float t[kTiny], w[kTiny], top = no_value(), sum = 0.0f;
    taught_all(a, r, at, t);
    uint32_t named = 0;  // bits of entries
#pragma unroll
    for (int i = 0; i < kTiny; ++i) {
        named |= at[i] >= 0 ? 1u << at[i] : 0;
        top = fmaxf(top, t[i]);
        w[i] = 0.0f;
    }
    s.live &= named != 0;
#pragma unroll
    for (int i = 0; i < kTiny; ++i) {
        if (i >= a.k)
            break;
        const float e = at[i] >= 0 ? exp2_whole((t[i] - top) * a.inv * kLog2e) : 0.0f;
        sum += e;
#pragma unroll
        for (int j = 0; j < kTiny; ++j)
            w[j] += j == at[i] ? e : 0.0f;
    }
    const float part = 1.0f / sum;
    T *dx = dlogits + r * dstride;
#pragma unroll
    for (int j = 0; j < kTiny; ++j) {
        if (j >= a.V)
            break;
        const float v = kMask && mask[j] == 0 ? no_value() : to_f32(x[j]);
        const float taken = named >> j & 1 ? w[j] * part : 0.0f;  // (part may be NaN)
        dx[j] = from_f32<T>(s.live && v != no_value() ? (share(s, v) - taken) * s.up : 0.0f);
    }
}

// ------------------------------------------------------------ host

// Threads of a row's block: 128 for many rows of up to 48 KB, 512 for few rows and those beyond 128 KB, else 256.  With 128,
// 256 and 512, rows of 16 bits: 4,864 of 2,000 10.4, 14.6 and 24.8 us, of 16,000 33.0, 37.0 and 50.0; 4,000 of 32,000 49.3,
// 47.3 and 54.8; 2,000 of 65,536 55.7, 49.4 and 49.9; 304 of 8,192 5.0, 4.8 and 6.0; 3,001 of 10,007 of 32 bits 23.0, 28.9
// and 35.3.
int threads_for(int64_t rows, int64_t bytes)
{
    if (rows < 152 || bytes > 131072)
        return 512;
    return bytes <= 49152 && rows >= 608 ? 128 : 256;
}

// Whether a row's gradient takes a warp, else blocks: 4,864 rows of 2,000 16-bit entries 10.4 us by warps and 24.7 by
// blocks, of 8,192 30.9 and 40.5; 304 of 8,192 10.5 and 6.4; 1,216 of 4,000 32-bit ones 10.4 and 8.8.
bool by_warps(int64_t rows, int64_t bytes) { return bytes <= 16384 && rows >= 1216; }

}  // namespace

cudaError_t launch_distill(const DistillArgs &a, const DistillOut &o, cudaStream_t st)
{
    with_type(a.dtype, [&](auto v) {
        using T = decltype(v);
        if (a.V > kTiny && a.V <= kNarrow) {
            with_lanes(a.V, [&](auto lanes, auto per) {
                auto run = [&](auto kernel) {
                    kernel<<<(unsigned)up(a.rows * lanes.value, kNarrowThreads), kNarrowThreads, 0, st>>>(a, o);
                };
                if (packs(a.logits, a.rows, a.V, a.stride, sizeof(T)))
                    run(distill_narrow_kernel<T, 16 / sizeof(T), lanes.value, per.value>);
                else
                    run(distill_narrow_kernel<T, 1, lanes.value, per.value>);
            });
            return;
        }
        with_flag(a.mask != nullptr, [&](auto mask) {
            if (a.V <= kTiny) {
                distill_tiny_kernel<T, mask.value><<<(unsigned)up(a.rows, kTinyThreads), kTinyThreads, 0, st>>>(a, o);
                return;
            }
            auto run = [&](auto kernel, int threads) {
                kernel<<<(unsigned)a.rows, threads, 0, st>>>(a, o);
            };
            const int threads = threads_for(a.rows, a.V * (int64_t)sizeof(T));
            if (threads == 128)
                run(distill_wide_kernel<T, 128, mask.value>, 128);
            else if (threads == 256)
                run(distill_wide_kernel<T, 256, mask.value>, 256);
            else
                run(distill_wide_kernel<T, 512, mask.value>, 512);
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_distill_grad(const DistillArgs &a, const float *dkl, const float *peak, const float *logz, void *dlogits,
                                int64_t dlogit_stride, cudaStream_t st)
{
    with_type(a.dtype, [&](auto v) {
        using T = decltype(v);
        T *dx = (T *)dlogits;
        const int64_t e = sizeof(T);
        if (a.V > kTiny && a.V <= kNarrow) {
            with_lanes(a.V, [&](auto lanes, auto per) {
                const int slots = kNarrowThreads / lanes.value;
                auto run = [&](auto kernel) {
                    kernel<<<(unsigned)up(a.rows, slots), kNarrowThreads, (size_t)slots * a.k * 8, st>>>(
                        a, dkl, peak, logz, dx, dlogit_stride);
                };
                if (packs(a.logits, a.rows, a.V, a.stride, e) && packs(dlogits, a.rows, a.V, dlogit_stride, e))
                    run(distill_narrow_grad_kernel<T, 16 / sizeof(T), lanes.value, per.value>);
                else
                    run(distill_narrow_grad_kernel<T, 1, lanes.value, per.value>);
            });
            return;
        }
        // whether dlogits' rows begin where in 16 bytes those of logits do
        const bool packed = ((reinterpret_cast<uintptr_t>(dlogits) ^ reinterpret_cast<uintptr_t>(a.logits)) & 15) == 0 &&
                            (a.rows <= 1 || (dlogit_stride - a.stride) * e % 16 == 0);
        with_flag(a.mask != nullptr, [&](auto mask) {
            if (a.V <= kTiny) {
                distill_tiny_grad_kernel<T, mask.value><<<(unsigned)up(a.rows, kTinyThreads), kTinyThreads, 0, st>>>(
                    a, dkl, peak, logz, dx, dlogit_stride);
            } else if (by_warps(a.rows, a.V * e)) {
                const int slots = kGradThreads / 32;
                distill_wide_grad_kernel<T, 32, mask.value>
                    <<<(unsigned)up(a.rows, slots), kGradThreads, (size_t)slots * a.k * 8, st>>>(a, dkl, peak, logz, dx,
                                                                                                 dlogit_stride, packed);
            } else {
                // parts of a row, of 32,768 entries: 4,000 rows of 32,000 16-bit ones take 88.6 us, in two 93.4; few rows in
                // twice as many: 1,000 of 65,536 49.2 us, and 51.5 so
                const int64_t parts = up(a.V, a.rows >= 1216 ? 32768 : 16384);
                distill_wide_grad_kernel<T, kGradThreads, mask.value>
                    <<<dim3((unsigned)a.rows, (unsigned)(parts < 65535 ? parts : 65535)), kGradThreads, (size_t)a.k * 8, st>>>(
                        a, dkl, peak, logz, dx, dlogit_stride, packed);
            }
        });
    });
    return cudaGetLastError();
}

}  // namespace av
