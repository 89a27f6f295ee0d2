// k_norm.cu -- layer norm of rows and its gradient.
//   forward   mean, var of a row, y = (x - mean) rstd w + b
//   backward  d = dy w; dx = rstd (d - mean(d) - xh mean(d xh)); dw = sum_rows dy xh; db = sum_rows dy
//
// Both are bound by memory: forward 2, backward 3 arrays of rows.  A row of up
// to 16,384 values is read once and stays in registers between its sums and
// its outputs.  A group of threads holds 8 to 32 values a thread: 2 to 32
// threads, or as many whole warps as the row fills, taken 16 bytes at a time
// where the rows allow it, the next row under way during this one where there
// are registers for it.  16-bit rows are bound by issue before they are bound
// by memory: they take more values a thread (the sums over a group cost some
// 30 instructions whatever it holds) and all arithmetic goes two values at a
// time.  Groups go from row to row with the parameters in shared memory and,
// backward, the running column sums in registers, so the weight's gradient
// costs no second pass: a block adds its groups' column sums in a fixed order,
// writes them once, and a second kernel adds the blocks'.  Longer rows are
// read again from L2 instead.
// The variance is the mean square of centred values: rows far from 0 lose
// nothing.
#include "async.cuh"
#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kSms = 152;
constexpr int kLongest = 16384;      // values of a row kept in registers
constexpr int kLongThreads = 512;    // for longer rows
constexpr int kColumns = 32;         // columns of a block that adds column sums
constexpr int kMostShared = 227 * 1024 - 2048;  // bytes a block asks for at most: what it can have beside its fixed arrays

// An array of parameters of either type, absent: `otherwise`.
__device__ __forceinline__ float param(const void *p, int type, int i, float otherwise)
{
    if (!p)
        return otherwise;
    return type == AV_F32    ? ((const float *)p)[i]
           : type == AV_BF16 ? to_f32(((const __nv_bfloat16 *)p)[i])
                             : to_f32(((const __half *)p)[i]);
}

__device__ __forceinline__ void put_param(void *p, int type, int i, float v)
{
    if (type == AV_F32)
        ((float *)p)[i] = v;
    else if (type == AV_BF16)
        ((__nv_bfloat16 *)p)[i] = from_f32<__nv_bfloat16>(v);
    else
        ((__half *)p)[i] = from_f32<__half>(v);
}

// kVec values at p: one load of 16 bytes, or one value.
template <class T, int kVec>
struct Pack {
    T v[kVec];
};

template <class T, int kVec>
__device__ __forceinline__ Pack<T, kVec> fetch(const T *p)
{
    Pack<T, kVec> r;
    if constexpr (kVec == 1)
        r.v[0] = *p;
    else
        *reinterpret_cast<uint4 *>(&r) = *reinterpret_cast<const uint4 *>(p);
    return r;
}

template <class T, int kVec>
__device__ __forceinline__ void put(T *p, const Pack<T, kVec> &r)
{
    if constexpr (kVec == 1)
        *p = r.v[0];
    else
        *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(&r);
}

// The threads of a row: kGroup of them (2 to 32), or, for kGroup 0, `size`
// threads of whole warps.
struct Group {
    int size, index, count, thread;  // index among the block's `count` groups, thread within the group
};
template <int kGroup>
__device__ __forceinline__ Group group_of(int size)
{
    Group g;
    g.size = kGroup ? kGroup : size;
    g.index = threadIdx.x / g.size;
    g.thread = threadIdx.x % g.size;
    g.count = blockDim.x / g.size;
    return g;
}

// Sums over a group, in all its threads, always in one order.  Groups of more
// than a warp pass their warps' sums through shared memory: two sets of slots
// in turn, so that one barrier a sum suffices.
template <int kGroup, int kN>
__device__ __forceinline__ void group_sum(float (&v)[kN], const Group &g, float (*slots)[32 * kN], int &turn)
{
#pragma unroll
    for (int o = (kGroup ? kGroup : 32) / 2; o; o >>= 1) {
#pragma unroll
        for (int k = 0; k < kN; ++k)
            v[k] += __shfl_xor_sync(~0u, v[k], o);
    }
    if (kGroup || g.size == 32)
        return;
    const int warp = threadIdx.x >> 5, first = warp - (g.thread >> 5), warps = g.size >> 5;
    float *s = slots[turn];
    turn ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int k = 0; k < kN; ++k)
            s[warp * kN + k] = v[k];
    }
    __syncwarp();
    asm volatile("bar.sync %0, %1;" ::"r"(g.index + 1), "r"(g.size) : "memory");
    if (warps <= 4) {
#pragma unroll
        for (int k = 0; k < kN; ++k)
            v[k] = s[first * kN + k] + s[(first + 1) * kN + k];
        if (warps > 2) {
#pragma unroll
            for (int k = 0; k < kN; ++k)
                v[k] += s[(first + 2) * kN + k] + (warps > 3 ? s[(first + 3) * kN + k] : 0.0f);
        }
        return;
    }
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < kN; ++k)
        v[k] = lane < warps ? s[(first + lane) * kN + k] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        if (o < warps) {
#pragma unroll
            for (int k = 0; k < kN; ++k)
                v[k] += __shfl_xor_sync(~0u, v[k], o);
        }
    }
#pragma unroll
    for (int k = 0; k < kN; ++k)
        v[k] = __shfl_sync(~0u, v[k], 0);
}

// A thread's packs of row r, zeros where there is nothing.
template <class T, int kVec, int kPacks>
__device__ __forceinline__ void fetch_row(Pack<T, kVec> (&q)[kPacks], const T *p, int64_t r, int64_t rows, int64_t stride,
                                          int at, int step, int n)
{
    const T *row = p + r * stride;
#pragma unroll
    for (int c = 0; c < kPacks; ++c) {
        const int i = c * step + at;
        if (r < rows && i < n)
            q[c] = fetch<T, kVec>(row + i);
        else
            q[c] = Pack<T, kVec>{};
    }
}

// Pairs of values: pair k of a thread is values 2k and 2k + 1 of its packs in
// order (of single values: of two packs).
template <class T, int kVec, int kPacks>
__device__ __forceinline__ float2 pair_of(const Pack<T, kVec> (&q)[kPacks], int k)
{
    return make_float2(to_f32(q[2 * k / kVec].v[2 * k % kVec]), to_f32(q[(2 * k + 1) / kVec].v[(2 * k + 1) % kVec]));
}

// Parameters in shared memory, a place a group's thread and value, four values
// (one, where rows are taken value by value) together.
template <int kVec, int kPer>
struct Params {
    static constexpr int kTogether = kVec == 1 ? 1 : 4;
    __device__ static __forceinline__ int at(int k, const Group &g)
    {
        return (k / kTogether * g.size + g.thread) * kTogether + k % kTogether;
    }
    __device__ static void load(float *to, const void *from, int type, int n, const Group &g, float otherwise)
    {
        if (g.index == 0) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int i = (k / kVec * g.size + g.thread) * kVec + k % kVec;
                to[at(k, g)] = i < n ? param(from, type, i, otherwise) : 0.0f;
            }
        }
    }
    __device__ static __forceinline__ float2 pair(const float *from, int k, const Group &g)
    {
        if constexpr (kVec == 1)
            return make_float2(from[at(2 * k, g)], from[at(2 * k + 1, g)]);
        else
            return *reinterpret_cast<const float2 *>(from + at(2 * k, g));
    }
};

// Rows in registers, the next one under way: 65,536 rows of 1,024 32-bit values
// 86 us, 6.2 TB/s; of 64 16-bit values 14 us, a sum over a group for every 64.
template <class T, int kVec, int kPer, int kGroup, int kMost, int kMin>
__global__ __launch_bounds__(kMost, kMin) void norm_kernel(int64_t rows, int n, int size, float eps, const T *x,
                                                           int64_t xs, const void *w, const void *b, int ptype, T *y,
                                                           int64_t ys, float *mean, float *rstd)
{
    constexpr int kPacks = kPer / kVec, kPairs = kPer / 2;
    using P = Params<kVec, kPer>;
    __shared__ float slots[2][32];
    extern __shared__ __align__(16) float shared[];
    int turn = 0;
    const Group g = group_of<kGroup>(size);
    const int at = g.thread * kVec, wide = g.size * kVec;
    float *sw = shared, *sb = shared + g.size * kPer;
    P::load(sw, w, ptype, n, g, 1.0f);
    P::load(sb, b, ptype, n, g, 0.0f);
    __syncthreads();
    const float per = 1.0f / n;
    const int64_t step = (int64_t)gridDim.x * g.count;
    int64_t r = (int64_t)blockIdx.x * g.count + g.index;
    Pack<T, kVec> next[kPacks];
    fetch_row<T, kVec>(next, x, r, rows, xs, at, wide, n);
    // (every group of a block goes round as often as its first, so that whole warps meet)
    for (int64_t r0 = (int64_t)blockIdx.x * g.count; r0 < rows; r0 += step, r += step) {
        float2 v[kPairs], t = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            v[k] = pair_of(next, k);
            t = add2(t, v[k]);
        }
        fetch_row<T, kVec>(next, x, r + step, rows, xs, at, wide, n);  // under way during this row
        float sum[1] = {t.x + t.y};
        group_sum<kGroup>(sum, g, slots, turn);
        const float m = sum[0] * per;
        const float2 less = make_float2(-m, -m);
        float square[1] = {0.0f};
        if constexpr (kVec == 1) {
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {
                v[k] = add2(v[k], less);
                square[0] += 2 * k * wide + at < n ? v[k].x * v[k].x : 0.0f;
                square[0] += (2 * k + 1) * wide + at < n ? v[k].y * v[k].y : 0.0f;
            }
        } else {
#pragma unroll
            for (int c = 0; c < kPacks; ++c) {
                t = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int k = c * kVec / 2; k < (c + 1) * kVec / 2; ++k) {
                    v[k] = add2(v[k], less);
                    t = fma2(v[k], v[k], t);
                }
                square[0] += c * wide + at < n ? t.x + t.y : 0.0f;
            }
        }
        group_sum<kGroup>(square, g, slots, turn);
        const float q = 1.0f / sqrtf(square[0] * per + eps);
        if (r >= rows)
            continue;
        T *out = y + r * ys;
#pragma unroll
        for (int c = 0; c < kPacks; ++c) {
            const int i = c * wide + at;
            Pack<T, kVec> o;
            if constexpr (kVec == 1) {
                const float z = c % 2 ? v[c / 2].y : v[c / 2].x;
                o.v[0] = from_f32<T>(fmaf(z * q, sw[P::at(c, g)], sb[P::at(c, g)]));
            } else {
#pragma unroll
                for (int e = 0; e < kVec; e += 2) {
                    const int k = (c * kVec + e) / 2;
                    const float2 z = fma2(mul2(v[k], make_float2(q, q)), P::pair(sw, k, g), P::pair(sb, k, g));
                    o.v[e] = from_f32<T>(z.x);
                    o.v[e + 1] = from_f32<T>(z.y);
                }
            }
            if (i < n)
                put<T, kVec>(out + i, o);
        }
        if (mean && g.thread == 0) {
            mean[r] = m;
            rstd[r] = q;
        }
    }
}

// dx, and each block's column sums to parts [block][2][n].  kHeld: these run in
// registers; in blocks of 1,024 threads, 64 registers each, in shared memory.
// 65,536 rows of 1,024 32-bit values 128 us with the columns' sums, 6.3 TB/s;
// 2,000 of 16,384 16-bit ones 98 us, 2.0 TB/s: one row at a time in a block.
template <class T, int kVec, int kPer, int kGroup, int kMost, int kMin, bool kAhead>
__global__ __launch_bounds__(kMost, kMin) void norm_grad_kernel(int64_t rows, int n, int size, const T *dy, int64_t dys,
                                                                const T *x, int64_t xs, const void *w, int ptype,
                                                                const float *mean, const float *rstd, T *dx,
                                                                int64_t dxs, float *parts)
{
    next_may_start();
    constexpr int kPacks = kPer / kVec, kPairs = kPer / 2;
    constexpr bool kHeld = kMost < 1024 || kPer <= 8;
    using P = Params<kVec, kPer>;
    __shared__ float slots[2][64];
    extern __shared__ __align__(16) float shared[];
    int turn = 0;
    const Group g = group_of<kGroup>(size);
    const int at = g.thread * kVec, wide = g.size * kVec, slot = blockDim.x;
    float *sw = shared, *running = shared + g.size * kPer;
    P::load(sw, w, ptype, n, g, 1.0f);
    const float2 none = make_float2(0.0f, 0.0f);
    float2 dw[kHeld ? kPairs : 1], db[kHeld ? kPairs : 1];
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        if constexpr (kHeld) {
            dw[k] = db[k] = none;
        } else {
            running[(2 * k) * slot + threadIdx.x] = running[(2 * k + 1) * slot + threadIdx.x] = 0.0f;
            running[(kPer + 2 * k) * slot + threadIdx.x] = running[(kPer + 2 * k + 1) * slot + threadIdx.x] = 0.0f;
        }
    }
    __syncthreads();
    const float per = 1.0f / n;
    const int64_t step = (int64_t)gridDim.x * g.count;
    int64_t r = (int64_t)blockIdx.x * g.count + g.index;
    Pack<T, kVec> xn[kPacks], dn[kPacks];
    float qn = 0.0f, mn = 0.0f;
    auto ahead = [&](int64_t row) {
        fetch_row<T, kVec>(xn, x, row, rows, xs, at, wide, n);
        fetch_row<T, kVec>(dn, dy, row, rows, dys, at, wide, n);
        qn = row < rows ? rstd[row] : 0.0f;
        mn = row < rows ? mean[row] : 0.0f;
    };
    if (kAhead)
        ahead(r);
    for (int64_t r0 = (int64_t)blockIdx.x * g.count; r0 < rows; r0 += step, r += step) {
        if (!kAhead)
            ahead(r);
        Pack<T, kVec> xp[kPacks], dp[kPacks];
#pragma unroll
        for (int c = 0; c < kPacks; ++c) {
            xp[c] = xn[c];
            dp[c] = dn[c];
        }
        const float q = qn;
        const float2 less = make_float2(-mn, -mn), scale = make_float2(q, q);
        if (kAhead)
            ahead(r + step);
        auto hat = [&](int k) { return mul2(add2(pair_of(xp, k), less), scale); };
        float2 s0 = none, s1 = none;
        // (past the row's end dy is 0, and with it all that is summed)
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            const float2 xh = hat(k), up = pair_of(dp, k), d = mul2(up, P::pair(sw, k, g));
            if constexpr (kHeld) {
                dw[k] = fma2(up, xh, dw[k]);
                db[k] = add2(db[k], up);
            } else {
                running[(2 * k) * slot + threadIdx.x] += up.x * xh.x;
                running[(2 * k + 1) * slot + threadIdx.x] += up.y * xh.y;
                running[(kPer + 2 * k) * slot + threadIdx.x] += up.x;
                running[(kPer + 2 * k + 1) * slot + threadIdx.x] += up.y;
            }
            s0 = add2(s0, d);
            s1 = fma2(d, xh, s1);
        }
        float s[2] = {s0.x + s0.y, s1.x + s1.y};
        group_sum<kGroup>(s, g, slots, turn);
        if (r >= rows)
            continue;
        const float2 a = make_float2(-s[0] * per * q, -s[0] * per * q), c1 = make_float2(-s[1] * per * q, -s[1] * per * q);
        T *out = dx + r * dxs;
#pragma unroll
        for (int c = 0; c < kPacks; c += kVec == 1 ? 2 : 1) {
            Pack<T, kVec> o[2];
#pragma unroll
            for (int e = 0; e < (kVec == 1 ? 2 : kVec); e += 2) {
                const int k = (c * kVec + e) / 2;
                const float2 d = mul2(pair_of(dp, k), P::pair(sw, k, g));
                const float2 z = fma2(hat(k), c1, fma2(d, scale, a));
                o[0].v[e % kVec] = from_f32<T>(z.x);
                o[kVec == 1].v[(e + 1) % kVec] = from_f32<T>(z.y);
            }
            if (c * wide + at < n)
                put<T, kVec>(out + c * wide + at, o[0]);
            if (kVec == 1 && (c + 1) * wide + at < n)
                put<T, kVec>(out + (c + 1) * wide + at, o[1]);
        }
    }
    if (!parts)
        return;
    float *mine = parts + (int64_t)blockIdx.x * 2 * n;
    auto column = [&](int k) { return k / kVec * wide + at + k % kVec; };
    if (g.count > 1) {
        if constexpr (kHeld) {
            if constexpr (kGroup > 0 && kGroup < 32) {  // groups of a warp first
#pragma unroll
                for (int o = kGroup; o < 32; o <<= 1) {
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) {
                        dw[k].x += __shfl_xor_sync(~0u, dw[k].x, o);
                        dw[k].y += __shfl_xor_sync(~0u, dw[k].y, o);
                        db[k].x += __shfl_xor_sync(~0u, db[k].x, o);
                        db[k].y += __shfl_xor_sync(~0u, db[k].y, o);
                    }
                }
            }
            const int team = kGroup && kGroup < 32 ? 32 : g.size, all = g.size * kPer;
            const bool speaks = threadIdx.x % team < g.size;
            float *sum = running;
            for (int t = 0; t < (int)blockDim.x / team; ++t) {
                if ((int)threadIdx.x / team == t && speaks) {
#pragma unroll
                    for (int k = 0; k < kPer; ++k) {
                        const int i = column(k);
                        sum[i] = (t ? sum[i] : 0.0f) + (k % 2 ? dw[k / 2].y : dw[k / 2].x);
                        sum[all + i] = (t ? sum[all + i] : 0.0f) + (k % 2 ? db[k / 2].y : db[k / 2].x);
                    }
                }
                __syncthreads();
            }
            for (int i = threadIdx.x; i < n; i += blockDim.x) {
                mine[i] = sum[i];
                mine[n + i] = sum[all + i];
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = column(k);
            if (i < n) {
                if constexpr (kHeld) {
                    mine[i] = k % 2 ? dw[k / 2].y : dw[k / 2].x;
                    mine[n + i] = k % 2 ? db[k / 2].y : db[k / 2].x;
                } else {
                    mine[i] = running[k * slot + threadIdx.x];
                    mine[n + i] = running[(kPer + k) * slot + threadIdx.x];
                }
            }
        }
    }
}

// ------------------------------------------------------------ rows by bulk copy

// Rows of whole warps come to shared memory whole, one copy a row and array,
// up to kDeep rows ahead of the one being taken: the bytes under way are not
// bound to registers.  A copy is of the 16-byte pieces that hold the row: those
// at its ends may hold a neighbour's bytes too, which nobody looks at.
constexpr int kDeep = 4;

// The rows that a group takes, in turn.
template <class T, int kArrays>
struct Ring {
    const T *from[kArrays];
    int64_t stride[kArrays];
    int64_t rows, step;
    int n, size;            // values of a row; bytes of a tile
    uint32_t tiles, bars;   // the group's tiles and barriers

    __device__ __forceinline__ uint32_t lead(int64_t r, int array) const
    {
        return (uint32_t)reinterpret_cast<uintptr_t>(from[array] + r * stride[array]) & 15u;
    }
    // Where row r's first value is.
    __device__ __forceinline__ uint32_t tile(int stage, int array, int64_t r) const
    {
        return tiles + (uint32_t)((stage * kArrays + array) * size) + lead(r, array);
    }
    // One thread: row r to the stage, if there is one.
    __device__ __forceinline__ void fetch(int64_t r, int stage) const
    {
        if (r >= rows)
            return;
        uint32_t bytes[kArrays], all = 0;
#pragma unroll
        for (int a = 0; a < kArrays; ++a) {
            bytes[a] = (lead(r, a) + n * (uint32_t)sizeof(T) + 15) & ~15u;
            all += bytes[a];
        }
        bar_expect(bars + 8 * stage, all);
#pragma unroll
        for (int a = 0; a < kArrays; ++a)
            bulk_load(tiles + (uint32_t)((stage * kArrays + a) * size),
                      reinterpret_cast<const char *>(from[a] + r * stride[a]) - lead(r, a), bytes[a], bars + 8 * stage);
    }
};
// Bytes of a tile for rows of n values of e bytes.
__host__ __device__ constexpr int tile_bytes(int n, int e) { return (n * e + 15 + 15) / 16 * 16; }

template <class T, int kVec>
__device__ __forceinline__ Pack<T, kVec> fetch_shared(uint32_t at)
{
    Pack<T, kVec> q;
    if constexpr (kVec == 1 && sizeof(T) == 4) {
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(*reinterpret_cast<float *>(&q)) : "r"(at) : "memory");
    } else if constexpr (kVec == 1) {
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(*reinterpret_cast<uint16_t *>(&q)) : "r"(at) : "memory");
    } else {
        uint4 &v = *reinterpret_cast<uint4 *>(&q);
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(at)
                     : "memory");
    }
    return q;
}

// A pair of values of consecutive places of packs o, to be stored at out.
template <class T, int kVec>
__device__ __forceinline__ void put_pairs(T *out, int at, int wide, int n, int c, Pack<T, kVec> (&o)[2])
{
    if (c * wide + at < n)
        put<T, kVec>(out + c * wide + at, o[0]);
    if (kVec == 1 && (c + 1) * wide + at < n)
        put<T, kVec>(out + (c + 1) * wide + at, o[1]);
}

// Rows by bulk copies, up to kDeep a group ahead, whatever they start on: 65,536
// rows of 1,024 16-bit values 43 us alone, 6.3 TB/s, at 2.5 of 4 instructions a
// cycle, and 55 one call after another, when the outputs before leave L2.
template <class T, int kVec, int kPer, int kMost, int kMin>
__global__ __launch_bounds__(kMost, kMin) void norm_ring_kernel(int64_t rows, int n, int size, float eps, const T *x,
                                                                int64_t xs, const void *w, const void *b, int ptype,
                                                                T *y, int64_t ys, float *mean, float *rstd, int deep)
{
    constexpr int kPacks = kPer / kVec, kPairs = kPer / 2;
    using P = Params<kVec, kPer>;
    __shared__ float slots[2][32];
    __shared__ uint64_t bars[kMost / 32 * kDeep];
    __shared__ int dead;
    extern __shared__ __align__(16) float shared[];
    int turn = 0;
    const Group g = group_of<0>(size);
    const int at = g.thread * kVec, wide = g.size * kVec;
    float *sw = shared, *sb = shared + g.size * kPer;
    Ring<T, 1> ring{{x}, {xs}, rows, (int64_t)gridDim.x * g.count, n, tile_bytes(n, sizeof(T)), 0, 0};
    ring.tiles = smem_addr(shared + 2 * g.size * kPer) + (uint32_t)(g.index * deep * ring.size);
    ring.bars = smem_addr(bars + g.index * kDeep);
    int64_t r = (int64_t)blockIdx.x * g.count + g.index;
    if (threadIdx.x == 0)
        dead = 0;
    if (g.thread == 0)
        for (int s = 0; s < deep; ++s)
            bar_init(ring.bars + 8 * s, 1);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    P::load(sw, w, ptype, n, g, 1.0f);
    P::load(sb, b, ptype, n, g, 0.0f);
    __syncthreads();
    if (g.thread == 0)
        for (int s = 0; s < deep; ++s)
            ring.fetch(r + s * ring.step, s);
    const float per = 1.0f / n;
    bool ok = true;
    int stage = 0, phase = 0;
    for (; r < rows; r += ring.step) {
        ok = ok && bar_wait(ring.bars + 8 * stage, phase, &dead);
        const uint32_t tile = ring.tile(stage, 0, r);
        float2 v[kPairs], t = make_float2(0.0f, 0.0f);
        Pack<T, kVec> p[kPacks];
#pragma unroll
        for (int c = 0; c < kPacks; ++c) {
            p[c] = Pack<T, kVec>{};
            if (c * wide + at < n)
                p[c] = fetch_shared<T, kVec>(tile + (uint32_t)((c * wide + at) * sizeof(T)));
        }
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            v[k] = pair_of(p, k);
            t = add2(t, v[k]);
        }
        float sum[1] = {t.x + t.y};
        if (!ok)  // (past a wait that ran out: no wrong row passes for a right one)
            sum[0] = __int_as_float(0x7fffffff);
        group_sum<0>(sum, g, slots, turn);
        if (g.thread == 0 && ok)  // (all of the group have read the row)
            ring.fetch(r + deep * ring.step, stage);
        if (++stage == deep) {
            stage = 0;
            phase ^= 1;
        }
        const float m = sum[0] * per;
        const float2 less = make_float2(-m, -m);
        float square[1] = {0.0f};
        if constexpr (kVec == 1) {
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {
                v[k] = add2(v[k], less);
                square[0] += 2 * k * wide + at < n ? v[k].x * v[k].x : 0.0f;
                square[0] += (2 * k + 1) * wide + at < n ? v[k].y * v[k].y : 0.0f;
            }
        } else {
#pragma unroll
            for (int c = 0; c < kPacks; ++c) {
                t = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int k = c * kVec / 2; k < (c + 1) * kVec / 2; ++k) {
                    v[k] = add2(v[k], less);
                    t = fma2(v[k], v[k], t);
                }
                square[0] += c * wide + at < n ? t.x + t.y : 0.0f;
            }
        }
        group_sum<0>(square, g, slots, turn);
        const float q = 1.0f / sqrtf(square[0] * per + eps);
        T *out = y + r * ys;
#pragma unroll
        for (int c = 0; c < kPacks; c += kVec == 1 ? 2 : 1) {
            Pack<T, kVec> o[2];
#pragma unroll
            for (int e = 0; e < (kVec == 1 ? 2 : kVec); e += 2) {
                const int k = (c * kVec + e) / 2;
                const float2 z = fma2(mul2(v[k], make_float2(q, q)), P::pair(sw, k, g), P::pair(sb, k, g));
                o[0].v[e % kVec] = from_f32<T>(z.x);
                o[kVec == 1].v[(e + 1) % kVec] = from_f32<T>(z.y);
            }
            put_pairs<T, kVec>(out, at, wide, n, c, o);
        }
        if (mean && g.thread == 0) {
            mean[r] = m;
            rstd[r] = q;
        }
    }
    if (!ok)
        linger();
}

// The same of x and dy: 74 us alone, 5.4 TB/s, and 80 one after another; warps
// wait at the groups' sums.
template <class T, int kVec, int kPer, int kMost, int kMin>
__global__ __launch_bounds__(kMost, kMin) void norm_grad_ring_kernel(int64_t rows, int n, int size, const T *dy,
                                                                     int64_t dys, const T *x, int64_t xs,
                                                                     const void *w, int ptype, const float *mean,
                                                                     const float *rstd, T *dx, int64_t dxs,
                                                                     float *parts, int deep)
{
    next_may_start();
    constexpr int kPacks = kPer / kVec, kPairs = kPer / 2;
    constexpr bool kKeep = sizeof(T) == 2 && kMin == 1;  // xh and d are kept: of 16 bits they are dear to make again
    using P = Params<kVec, kPer>;
    __shared__ float slots[2][64];
    __shared__ uint64_t bars[kMost / 32 * kDeep];
    __shared__ int dead;
    extern __shared__ __align__(16) float shared[];
    int turn = 0;
    const Group g = group_of<0>(size);
    const int at = g.thread * kVec, wide = g.size * kVec;
    float *sw = shared;
    Ring<T, 2> ring{{x, dy}, {xs, dys}, rows, (int64_t)gridDim.x * g.count, n, tile_bytes(n, sizeof(T)), 0, 0};
    ring.tiles = smem_addr(shared + g.size * kPer) + (uint32_t)(g.index * deep * 2 * ring.size);
    ring.bars = smem_addr(bars + g.index * kDeep);
    int64_t r = (int64_t)blockIdx.x * g.count + g.index;
    if (threadIdx.x == 0)
        dead = 0;
    if (g.thread == 0)
        for (int s = 0; s < deep; ++s)
            bar_init(ring.bars + 8 * s, 1);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    P::load(sw, w, ptype, n, g, 1.0f);
    __syncthreads();
    if (g.thread == 0)
        for (int s = 0; s < deep; ++s)
            ring.fetch(r + s * ring.step, s);
    const float2 none = make_float2(0.0f, 0.0f);
    float2 dw[kPairs], db[kPairs];
#pragma unroll
    for (int k = 0; k < kPairs; ++k)
        dw[k] = db[k] = none;
    const float per = 1.0f / n;
    float q_next = r < rows ? rstd[r] : 0.0f, m_next = r < rows ? mean[r] : 0.0f;
    bool ok = true;
    int stage = 0, phase = 0;
    for (; r < rows; r += ring.step) {
        const float q = q_next;
        const float2 less = make_float2(-m_next, -m_next), scale = make_float2(q, q);
        const bool more = r + ring.step < rows;
        q_next = more ? rstd[r + ring.step] : 0.0f;
        m_next = more ? mean[r + ring.step] : 0.0f;
        ok = ok && bar_wait(ring.bars + 8 * stage, phase, &dead);
        const uint32_t xt = ring.tile(stage, 0, r), dt = ring.tile(stage, 1, r);
        Pack<T, kVec> xp[kPacks], dp[kPacks];
#pragma unroll
        for (int c = 0; c < kPacks; ++c) {
            xp[c] = dp[c] = Pack<T, kVec>{};
            if (c * wide + at < n) {
                xp[c] = fetch_shared<T, kVec>(xt + (uint32_t)((c * wide + at) * sizeof(T)));
                dp[c] = fetch_shared<T, kVec>(dt + (uint32_t)((c * wide + at) * sizeof(T)));
            }
        }
        float2 kept_hat[kKeep ? kPairs : 1], kept_d[kKeep ? kPairs : 1];
        auto hat = [&](int k) { return mul2(add2(pair_of(xp, k), less), scale); };
        float2 s0 = none, s1 = none;
        // (past the row's end dy is 0, and with it all that is summed)
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            const float2 xh = hat(k), up = pair_of(dp, k), d = mul2(up, P::pair(sw, k, g));
            dw[k] = fma2(up, xh, dw[k]);
            db[k] = add2(db[k], up);
            if constexpr (kKeep) {
                kept_hat[k] = xh;
                kept_d[k] = d;
            }
            s0 = add2(s0, d);
            s1 = fma2(d, xh, s1);
        }
        float s[2] = {s0.x + s0.y, s1.x + s1.y};
        if (!ok)
            s[0] = __int_as_float(0x7fffffff);
        group_sum<0>(s, g, slots, turn);
        if (g.thread == 0 && ok)
            ring.fetch(r + deep * ring.step, stage);
        if (++stage == deep) {
            stage = 0;
            phase ^= 1;
        }
        const float2 a = make_float2(-s[0] * per * q, -s[0] * per * q), c1 = make_float2(-s[1] * per * q, -s[1] * per * q);
        T *out = dx + r * dxs;
#pragma unroll
        for (int c = 0; c < kPacks; c += kVec == 1 ? 2 : 1) {
            Pack<T, kVec> o[2];
#pragma unroll
            for (int e = 0; e < (kVec == 1 ? 2 : kVec); e += 2) {
                const int k = (c * kVec + e) / 2;
                const float2 d = kKeep ? kept_d[kKeep ? k : 0] : mul2(pair_of(dp, k), P::pair(sw, k, g));
                const float2 z = fma2(kKeep ? kept_hat[kKeep ? k : 0] : hat(k), c1, fma2(d, scale, a));
                o[0].v[e % kVec] = from_f32<T>(z.x);
                o[kVec == 1].v[(e + 1) % kVec] = from_f32<T>(z.y);
            }
            put_pairs<T, kVec>(out, at, wide, n, c, o);
        }
    }
    if (!ok) {
        linger();
#pragma unroll
        for (int k = 0; k < kPairs; ++k)
            dw[k] = db[k] = make_float2(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff));
    }
    if (!parts)
        return;
    // the groups' sums, in order, on the way out (the tiles are done with)
    __syncthreads();
    float *mine = parts + (int64_t)blockIdx.x * 2 * n, *sum = shared + g.size * kPer;
    const int all = g.size * kPer;
    for (int t = 0; t < g.count; ++t) {
        if (g.index == t) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const int i = k / kVec * wide + at + k % kVec;
                const float a = k % 2 ? dw[k / 2].y : dw[k / 2].x, c = k % 2 ? db[k / 2].y : db[k / 2].x;
                sum[i] = (t ? sum[i] : 0.0f) + a;
                sum[all + i] = (t ? sum[all + i] : 0.0f) + c;
            }
        }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        mine[i] = sum[i];
        mine[n + i] = sum[all + i];
    }
}

// ------------------------------------------------------------ longer rows

__device__ float long_sum(float v, float *s)
{
    for (int o = 16; o; o >>= 1)
        v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        s[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
    for (int i = 0; i < kLongThreads / 32; ++i)
        t += s[i];
    return t;
}

// A block a row, read three times, twice from L2 (counted down: the last step
// up of a row of 2^31 - 1 values would go beyond an int): 1,500 rows of 20,011 16-bit
// values 79 us, the gradient with the columns' sums 202.
template <class T>
__global__ __launch_bounds__(kLongThreads) void norm_long_kernel(int64_t rows, int n, float eps, const T *x, int64_t xs,
                                                                 const void *w, const void *b, int ptype, T *y,
                                                                 int64_t ys, float *mean, float *rstd)
{
    __shared__ float s[kLongThreads / 32];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + r * xs;
        float v = 0.0f;
#pragma unroll 8
        for (int left = n - (int)threadIdx.x; left > 0; left -= kLongThreads)
            v += to_f32(xr[n - left]);
        const float m = long_sum(v, s) / n;
        v = 0.0f;
#pragma unroll 8
        for (int left = n - (int)threadIdx.x; left > 0; left -= kLongThreads) {
            const int i = n - left;
            const float c = to_f32(xr[i]) - m;
            v += c * c;
        }
        const float q = 1.0f / sqrtf(long_sum(v, s) / n + eps);
#pragma unroll 8
        for (int left = n - (int)threadIdx.x; left > 0; left -= kLongThreads) {
            const int i = n - left;
            y[r * ys + i] = from_f32<T>((to_f32(xr[i]) - m) * q * param(w, ptype, i, 1.0f) + param(b, ptype, i, 0.0f));
        }
        if (mean && threadIdx.x == 0) {
            mean[r] = m;
            rstd[r] = q;
        }
    }
}

template <class T>
__global__ __launch_bounds__(kLongThreads) void norm_long_dx_kernel(int64_t rows, int n, const T *dy, int64_t dys,
                                                                    const T *x, int64_t xs, const void *w, int ptype,
                                                                    const float *mean, const float *rstd, T *dx,
                                                                    int64_t dxs)
{
    __shared__ float s[kLongThreads / 32];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + r * xs, *dr = dy + r * dys;
        const float m = mean[r], q = rstd[r];
        float a = 0.0f, c = 0.0f;
#pragma unroll 8
        for (int left = n - (int)threadIdx.x; left > 0; left -= kLongThreads) {
            const int i = n - left;
            const float d = to_f32(dr[i]) * param(w, ptype, i, 1.0f);
            a += d;
            c += d * (to_f32(xr[i]) - m) * q;
        }
        a = long_sum(a, s) / n;
        c = long_sum(c, s) / n;
#pragma unroll 8
        for (int left = n - (int)threadIdx.x; left > 0; left -= kLongThreads) {
            const int i = n - left;
            const float d = to_f32(dr[i]) * param(w, ptype, i, 1.0f);
            dx[r * dxs + i] = from_f32<T>(q * (d - a - (to_f32(xr[i]) - m) * q * c));
        }
    }
}

// Column sums of a block's share of the rows: 32 columns, eight rows at a time.
template <class T>
__global__ __launch_bounds__(256) void norm_long_columns_kernel(int64_t rows, int n, const T *dy, int64_t dys,
                                                                const T *x, int64_t xs, const float *mean,
                                                                const float *rstd, float *parts)
{
    next_may_start();
    __shared__ float s[2][8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    const int64_t r0 = rows * blockIdx.y / gridDim.y, r1 = rows * (blockIdx.y + 1) / gridDim.y;
    float a = 0.0f, c = 0.0f;
    if (i < n) {
#pragma unroll 4
        for (int64_t r = r0 + warp; r < r1; r += 8) {
            const float d = to_f32(dy[r * dys + i]);
            a += d * (to_f32(x[r * xs + i]) - mean[r]) * rstd[r];
            c += d;
        }
    }
    s[0][warp][lane] = a;
    s[1][warp][lane] = c;
    __syncthreads();
    if (warp != 0 || i >= n)
        return;
    for (int k = 1; k < 8; ++k) {
        a += s[0][k][lane];
        c += s[1][k][lane];
    }
    parts[(int64_t)blockIdx.y * 2 * n + i] = a;
    parts[(int64_t)blockIdx.y * 2 * n + n + i] = c;
}

// dw, db: the blocks' column sums, 32 columns of either a block.
__global__ __launch_bounds__(256) void norm_columns_kernel(int count, int n, const float *parts, int ptype, void *dw,
                                                           void *db)
{
    __shared__ float s[8][kColumns];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * kColumns + lane;
    const float *from = parts + (blockIdx.y ? n : 0);
    void *to = blockIdx.y ? db : dw;
    after_previous();
    if (!to)
        return;
    float v = 0.0f;
    if (i < n) {
#pragma unroll 8
        for (int g = warp; g < count; g += 8)
            v += from[(int64_t)g * 2 * n + i];
    }
    s[warp][lane] = v;
    __syncthreads();
    if (warp != 0 || i >= n)
        return;
    for (int k = 1; k < 8; ++k)
        v += s[k][lane];
    put_param(to, ptype, i, v);
}

// ------------------------------------------------------------ host

// How rows of n values are taken: values a thread, threads a group (up to 32,
// or whole warps), threads a block, blocks an SM.
struct Shape {
    int per, group, block, most, resident;
};

// most, resident: the kernel's bounds; blocks of several groups are of up to
// `several` threads.
Shape shape_for(int n, int per, int several, int most, int resident)
{
    Shape s;
    s.per = per;
    s.group = 2;
    while (s.group < 32 && s.group * per < n)
        s.group *= 2;
    if (s.group * per < n)
        s.group = (n + 32 * per - 1) / (32 * per) * 32;
    s.block = s.group > several ? s.group : several / s.group * s.group;
    s.most = most;
    s.resident = resident;
    return s;
}

// Rows that go through registers: those that are not `ringed`.  wide: 16-bit
// values, eight at a time.
Shape shape_of(int n, bool wide, bool back)
{
    if (n > 1024)
        return shape_for(n, 16, 1024, 1024, 1);
    if (wide && n > 32)
        return back ? shape_for(n, 16, 512, 512, 1) : shape_for(n, 32, 256, 256, 3);
    return shape_for(n, 8, 512, 512, 2);
}

// Whether rows go by bulk copies: where these are of a kilobyte or more (a group
// is of whole warps then).  Through registers 32,768 rows of 1,024 16-bit values
// take 55 us and by copies 31, 65,536 of 1,001 32-bit ones, which do not start
// on 16 bytes, 131 and 103; but those of 1,024, in whole packs, 86 and 99 (the
// gradient 128 and 130, of 384 136 and 150).
bool ringed(int n, int e, bool wide, bool back)
{
    return n * e > 1024 && !(e == 4 && wide && n <= 1024) && n <= (back ? 8192 : kLongest);
}
Shape ring_of(int n, bool wide, bool back)
{
    if (back)
        return wide || n > 4096 ? shape_for(n, 16, 512, 512, 1) : shape_for(n, 8, 512, 512, 2);
    if (n > 8192)
        return shape_for(n, 16, 1024, 1024, 1);
    if (n > 4096)
        return shape_for(n, 16, 512, 512, 2);
    return wide ? shape_for(n, 32, 256, 256, 3) : shape_for(n, 8, 512, 512, 2);
}
// Shared memory of a block: the parameters, and `deep` rows a group: as many,
// up to kDeep, as leave room for the blocks that an SM can hold, or for one.
struct Room {
    int deep, bytes, resident;
};
Room room_of(const Shape &s, int n, int e, bool back)
{
    const int fixed = (back ? 1 : 2) * s.per * s.group * 4, row = s.block / s.group * (back ? 2 : 1) * tile_bytes(n, e);
    const int sums = back ? 2 * s.per * s.group * 4 : 0;  // (over the rows' tiles)
    Room m{};
    for (m.resident = s.resident; m.resident > 0; --m.resident) {
        m.deep = ((kMostShared + 2048) / m.resident - 2048 - fixed) / row;
        if (m.deep >= (m.resident > 1 ? 3 : 1))
            break;
    }
    m.deep = m.deep > kDeep ? kDeep : m.deep;
    m.bytes = fixed + (m.deep * row > sums ? m.deep * row : sums);
    return m;
}

// Blocks of a launch: as many as the GPU holds at once, or what there is to do.
int blocks_of(int64_t rows, int n, int e, bool wide, bool back)
{
    if (n > kLongest)
        return (int)(rows < 4 * kSms ? rows : 4 * kSms);
    const bool eights = wide && e == 2, ring = ringed(n, e, wide, back);
    const Shape s = ring ? ring_of(n, eights, back) : shape_of(n, eights, back);
    const int64_t need = (rows + s.block / s.group - 1) / (s.block / s.group),
                  most = kSms * (ring ? room_of(s, n, e, back).resident : s.resident);
    return (int)(need < most ? need : most);
}

// Rows' parts of the column sums of long rows: blocks for every SM, eight rows each at least.
int long_parts(int64_t rows, int n)
{
    const int64_t slabs = ((int64_t)n + 31) / 32, want = (8 * kSms + slabs - 1) / slabs, most = (rows + 7) / 8;
    return (int)(want < most ? want : most);
}

int parts_of(int64_t rows, int n, int e, bool wide)
{
    return n > kLongest ? long_parts(rows, n) : blocks_of(rows, n, e, wide, true);
}

// Rows that start on 16 bytes and hold whole packs of them.
bool packs(int64_t rows, int n, int e, const void *p, int64_t stride)
{
    return n % (16 / e) == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (rows <= 1 || stride * e % 16 == 0);
}

// Lets a kernel have what any of its launches asks for: the limit is the
// kernel's and not the call's, so that calls from several threads all set the same.
template <class K>
cudaError_t let_share(K kernel)
{
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
}

// Calls f with a shape's values a thread, threads a group (0: whole warps),
// threads a block at most and blocks an SM as constants.
template <int kPer, int kMost, int kMin, class F>
void with_group(const Shape &s, F f)
{
    using std::integral_constant;
    const integral_constant<int, kPer> per;
    const integral_constant<int, kMost> most;
    const integral_constant<int, kMin> resident;
    if (s.group == 2)
        f(per, integral_constant<int, 2>(), most, resident);
    else if (s.group == 4)
        f(per, integral_constant<int, 4>(), most, resident);
    else if (s.group == 8)
        f(per, integral_constant<int, 8>(), most, resident);
    else if (s.group == 16)
        f(per, integral_constant<int, 16>(), most, resident);
    else
        f(per, integral_constant<int, 0>(), most, resident);
}
template <int kPer, int kMost, int kMin, class F>
void whole_warps(F f)
{
    using std::integral_constant;
    f(integral_constant<int, kPer>(), integral_constant<int, 0>(), integral_constant<int, kMost>(),
      integral_constant<int, kMin>());
}
template <bool kBack, bool kEights, class F>
void with_shape(const Shape &s, F f)
{
    if constexpr (kBack) {
        if (s.most == 1024)
            return whole_warps<16, 1024, 1>(f);
        if constexpr (kEights) {
            if (s.per == 16)
                return with_group<16, 512, 1>(s, f);
        }
    } else if constexpr (kEights) {
        if (s.per == 32)
            return with_group<32, 256, 3>(s, f);
    }
    with_group<8, 512, 2>(s, f);
}

}  // namespace

// (of whatever type and alignment: the most)
int64_t norm_work_bytes(int64_t rows, int n)
{
    int most = 0;
    for (int k = 0; k < 4; ++k) {
        const int parts = parts_of(rows, n, k & 1 ? 4 : 2, k >> 1);
        most = parts > most ? parts : most;
    }
    return (int64_t)most * 2 * n * 4;
}

cudaError_t launch_norm(int64_t rows, int n, int dtype, int param_dtype, float eps, const void *x, int64_t x_stride,
                        const void *weight, const void *bias, void *y, int64_t y_stride, float *mean, float *rstd,
                        cudaStream_t st)
{
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int kWide = 16 / sizeof(T);
        const bool wide = packs(rows, n, sizeof(T), x, x_stride) && packs(rows, n, sizeof(T), y, y_stride);
        const bool eights = wide && sizeof(T) == 2;
        const int blocks = blocks_of(rows, n, sizeof(T), wide, false);
        if (n > kLongest) {
            norm_long_kernel<T><<<blocks, kLongThreads, 0, st>>>(rows, n, eps, (const T *)x, x_stride, weight, bias,
                                                                 param_dtype, (T *)y, y_stride, mean, rstd);
            return cudaGetLastError();
        }
        cudaError_t e = cudaSuccess;
        if (ringed(n, sizeof(T), wide, false)) {
            const Shape s = ring_of(n, eights, false);
            const Room room = room_of(s, n, sizeof(T), false);
            auto run = [&](auto kernel) {
                e = let_share(kernel);
                if (e == cudaSuccess)
                    kernel<<<blocks, s.block, room.bytes, st>>>(rows, n, s.group, eps, (const T *)x, x_stride, weight,
                                                                bias, param_dtype, (T *)y, y_stride, mean, rstd,
                                                                room.deep);
            };
            auto by = [&](auto vec) {
                if (s.most == 1024)
                    return run(norm_ring_kernel<T, vec.value, 16, 1024, 1>);
                if (s.per == 16)
                    return run(norm_ring_kernel<T, vec.value, 16, 512, 2>);
                if constexpr (vec.value == 8)
                    run(norm_ring_kernel<T, 8, 32, 256, 3>);
                else
                    run(norm_ring_kernel<T, vec.value, 8, 512, 2>);
            };
            if (wide)
                by(std::integral_constant<int, kWide>());
            else
                by(std::integral_constant<int, 1>());
            return e != cudaSuccess ? e : cudaGetLastError();
        }
        const Shape s = shape_of(n, eights, false);
        const int shared = 2 * s.per * s.group * 4;
        auto run = [&](auto kernel) {
            if (shared > 40 * 1024)
                e = let_share(kernel);
            if (e == cudaSuccess)
                kernel<<<blocks, s.block, shared, st>>>(rows, n, s.group, eps, (const T *)x, x_stride, weight, bias,
                                                        param_dtype, (T *)y, y_stride, mean, rstd);
        };
        auto packed = [&](auto per, auto group, auto most, auto least) {
            run(norm_kernel<T, kWide, per.value, group.value, most.value, least.value>);
        };
        auto single = [&](auto per, auto group, auto most, auto least) {
            run(norm_kernel<T, 1, per.value, group.value, most.value, least.value>);
        };
        if (wide)
            with_shape<false, sizeof(T) == 2>(s, packed);
        else
            with_shape<false, false>(s, single);
        return e != cudaSuccess ? e : cudaGetLastError();
    });
}

cudaError_t launch_norm_grad(int64_t rows, int n, int dtype, int param_dtype, const void *dy, int64_t dy_stride,
                             const void *x, int64_t x_stride, const void *weight, const float *mean,
                             const float *rstd, void *dx, int64_t dx_stride, void *dweight, void *dbias, void *work,
                             cudaStream_t st)
{
    const bool sums = dweight || dbias;
    const int e_bytes = dtype == AV_F32 ? 4 : 2;
    const bool wide = packs(rows, n, e_bytes, x, x_stride) && packs(rows, n, e_bytes, dy, dy_stride) &&
                      packs(rows, n, e_bytes, dx, dx_stride);
    const bool eights = wide && e_bytes == 2;
    const int count = parts_of(rows, n, e_bytes, wide);
    float *parts = (float *)work;
    cudaError_t e = cudaSuccess;
    if (rows > 0) {
        e = with_type(dtype, [&](auto t) {
            using T = decltype(t);
            constexpr int kWide = 16 / sizeof(T);
            const int blocks = blocks_of(rows, n, sizeof(T), wide, true);
            if (n > kLongest) {
                norm_long_dx_kernel<T><<<blocks, kLongThreads, 0, st>>>(rows, n, (const T *)dy, dy_stride,
                                                                        (const T *)x, x_stride, weight, param_dtype,
                                                                        mean, rstd, (T *)dx, dx_stride);
                if (sums)
                    norm_long_columns_kernel<T><<<dim3((unsigned)(((int64_t)n + 31) / 32), count), 256, 0, st>>>(
                        rows, n, (const T *)dy, dy_stride, (const T *)x, x_stride, mean, rstd, parts);
                return cudaGetLastError();
            }
            cudaError_t bad = cudaSuccess;
            if (ringed(n, sizeof(T), wide, true)) {
                const Shape s = ring_of(n, eights, true);
                const Room room = room_of(s, n, sizeof(T), true);
                auto run = [&](auto kernel) {
                    bad = let_share(kernel);
                    if (bad == cudaSuccess)
                        kernel<<<blocks, s.block, room.bytes, st>>>(rows, n, s.group, (const T *)dy, dy_stride,
                                                                    (const T *)x, x_stride, weight, param_dtype, mean,
                                                                    rstd, (T *)dx, dx_stride, sums ? parts : nullptr,
                                                                    room.deep);
                };
                if constexpr (sizeof(T) == 2) {
                    if (eights)
                        run(norm_grad_ring_kernel<T, 8, 16, 512, 1>);
                    else
                        s.per == 8 ? run(norm_grad_ring_kernel<T, 1, 8, 512, 2>) : run(norm_grad_ring_kernel<T, 1, 16, 512, 1>);
                } else if (wide) {
                    s.per == 8 ? run(norm_grad_ring_kernel<T, 4, 8, 512, 2>) : run(norm_grad_ring_kernel<T, 4, 16, 512, 1>);
                } else {
                    s.per == 8 ? run(norm_grad_ring_kernel<T, 1, 8, 512, 2>) : run(norm_grad_ring_kernel<T, 1, 16, 512, 1>);
                }
                return bad != cudaSuccess ? bad : cudaGetLastError();
            }
            const Shape s = shape_of(n, eights, true);
            // the weight; running sums, or the groups' sums on their way together
            const int sums_at = s.most == 1024 ? 2 * s.per * s.block : s.block > s.group ? 2 * s.per * s.group : 0;
            const int shared = (s.per * s.group + sums_at) * 4;
            auto run = [&](auto kernel) {
                if (shared > 40 * 1024)
                    bad = let_share(kernel);
                if (bad == cudaSuccess)
                    kernel<<<blocks, s.block, shared, st>>>(rows, n, s.group, (const T *)dy, dy_stride, (const T *)x,
                                                            x_stride, weight, param_dtype, mean, rstd, (T *)dx,
                                                            dx_stride, sums ? parts : nullptr);
            };
            // (the next row goes ahead where a thread has 128 registers)
            auto packed = [&](auto per, auto group, auto most, auto least) {
                run(norm_grad_kernel<T, kWide, per.value, group.value, most.value, least.value, most.value == 512 && least.value == 1>);
            };
            auto single = [&](auto per, auto group, auto most, auto least) {
                run(norm_grad_kernel<T, 1, per.value, group.value, most.value, least.value, false>);
            };
            if (wide)
                with_shape<true, sizeof(T) == 2>(s, packed);
            else
                with_shape<true, false>(s, single);
            return bad != cudaSuccess ? bad : cudaGetLastError();
        });
        if (e != cudaSuccess)
            return e;
    }
    if (sums)
        return launch_chained(norm_columns_kernel, dim3((unsigned)(((int64_t)n + kColumns - 1) / kColumns), 2), 256, 0, st, rows > 0, count, n,
                              parts, param_dtype, dweight, dbias);
    return cudaSuccess;
}

}  // namespace av
