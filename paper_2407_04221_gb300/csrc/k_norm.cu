// k_norm.cu -- layer norm of rows and its gradient.
//   forward   mean, var of a row, y = (x - mean) rstd w + b
//   backward  d = dy w; dx = rstd (d - mean(d) - xh mean(d xh)); dw = sum_rows dy xh; db = sum_rows dy
//
// Both are bound by memory: forward 2, backward 3 arrays of rows.  A row of up
// to 16,384 values is read once and stays in registers between its sums and
// its outputs.  A group of threads holds 16 values a thread (8 of 32 bits): 2
// to 32 threads, or as many whole warps as the row fills, taken 16 bytes at a
// time where the rows allow it, the next row under way during this one.
// Groups go from row to row with the weight (and, backward, the running column
// sums) at hand, so the weight's gradient costs no second pass: a block adds
// its groups' column sums in a fixed order, writes them once, and a second
// kernel adds the blocks'.  Longer rows are read again from L2 instead.
// The variance is the mean square of centred values: rows far from 0 lose
// nothing.
#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kSms = 152;
constexpr int kBlock = 512;          // threads of a block of several groups
constexpr int kLongest = 16384;      // values of a row kept in registers
constexpr int kLongThreads = 512;    // for longer rows
constexpr int kColumns = 32;         // columns of a block that adds column sums

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

// kMost: threads of a block at most.  1,024 leave 64 registers a thread: there
// the parameters (and, backward, the running sums) live in shared memory, a
// slot a thread and value, and no row is fetched ahead.
template <class T, int kVec, int kPer, int kGroup, int kMost>
__global__ __launch_bounds__(kMost, 1) void norm_kernel(int64_t rows, int n, int size, float eps, const T *x, int64_t xs,
                                                        const void *w, const void *b, int ptype, T *y, int64_t ys,
                                                        float *mean, float *rstd)
{
    constexpr int kPacks = kPer / kVec;
    constexpr bool kHeld = kMost < 1024;
    __shared__ float slots[2][32];
    extern __shared__ float shared[];
    int turn = 0;
    const Group g = group_of<kGroup>(size);
    const int at = g.thread * kVec, wide = g.size * kVec, slot = blockDim.x;
    float wv[kHeld ? kPer : 1], bv[kHeld ? kPer : 1];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int i = k / kVec * wide + at + k % kVec;
        const float wk = i < n ? param(w, ptype, i, 1.0f) : 0.0f, bk = i < n ? param(b, ptype, i, 0.0f) : 0.0f;
        if constexpr (kHeld) {
            wv[k] = wk;
            bv[k] = bk;
        } else {
            shared[k * slot + threadIdx.x] = wk;
            shared[(kPer + k) * slot + threadIdx.x] = bk;
        }
    }
    const float per = 1.0f / n;
    const int64_t step = (int64_t)gridDim.x * g.count;
    int64_t r = (int64_t)blockIdx.x * g.count + g.index;
    Pack<T, kVec> next[kPacks];
    fetch_row<T, kVec>(next, x, r, rows, xs, at, wide, n);
    // (every group of a block goes round as often as its first, so that whole warps meet)
    for (int64_t r0 = (int64_t)blockIdx.x * g.count; r0 < rows; r0 += step, r += step) {
        float v[kPer];
        float sum[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            v[k] = to_f32(next[k / kVec].v[k % kVec]);
            sum[0] += v[k];
        }
        fetch_row<T, kVec>(next, x, r + step, rows, xs, at, wide, n);  // under way during this row
        group_sum<kGroup>(sum, g, slots, turn);
        const float m = sum[0] * per;
        float square[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < kPacks; ++c) {
            float t = 0.0f;
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                v[c * kVec + k] -= m;
                t += v[c * kVec + k] * v[c * kVec + k];
            }
            square[0] += c * wide + at < n ? t : 0.0f;
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
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const int k = c * kVec + e;
                const float wk = kHeld ? wv[kHeld ? k : 0] : shared[k * slot + threadIdx.x];
                const float bk = kHeld ? bv[kHeld ? k : 0] : shared[(kPer + k) * slot + threadIdx.x];
                o.v[e] = from_f32<T>(v[k] * q * wk + bk);
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

// dx, and each block's column sums to parts [block][2][n].
template <class T, int kVec, int kPer, int kGroup, int kMost>
__global__ __launch_bounds__(kMost, 1) void norm_grad_kernel(int64_t rows, int n, int size, const T *dy, int64_t dys,
                                                             const T *x, int64_t xs, const void *w, int ptype,
                                                             const float *mean, const float *rstd, T *dx, int64_t dxs,
                                                             float *parts)
{
    constexpr int kPacks = kPer / kVec;
    constexpr bool kHeld = kMost < 1024;
    __shared__ float slots[2][64];
    extern __shared__ float shared[];
    int turn = 0;
    const Group g = group_of<kGroup>(size);
    const int at = g.thread * kVec, wide = g.size * kVec, slot = blockDim.x;
    float wv[kHeld ? kPer : 1], dw[kHeld ? kPer : 1] = {}, db[kHeld ? kPer : 1] = {};
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int i = k / kVec * wide + at + k % kVec;
        const float wk = i < n ? param(w, ptype, i, 1.0f) : 0.0f;
        if constexpr (kHeld) {
            wv[k] = wk;
        } else {
            shared[k * slot + threadIdx.x] = wk;
            shared[(kPer + k) * slot + threadIdx.x] = shared[(2 * kPer + k) * slot + threadIdx.x] = 0.0f;
        }
    }
    const float per = 1.0f / n;
    const int64_t step = (int64_t)gridDim.x * g.count;
    int64_t r = (int64_t)blockIdx.x * g.count + g.index;
    Pack<T, kVec> xn[kPacks], dn[kPacks];
    float qn = 0.0f, mn = 0.0f;
    auto ahead = [&](int64_t at_row) {
        fetch_row<T, kVec>(xn, x, at_row, rows, xs, at, wide, n);
        fetch_row<T, kVec>(dn, dy, at_row, rows, dys, at, wide, n);
        qn = at_row < rows ? rstd[at_row] : 0.0f;
        mn = at_row < rows ? mean[at_row] : 0.0f;
    };
    if constexpr (kHeld)
        ahead(r);
    for (int64_t r0 = (int64_t)blockIdx.x * g.count; r0 < rows; r0 += step, r += step) {
        Pack<T, kVec> xp[kPacks], dp[kPacks];
        if constexpr (!kHeld)
            ahead(r);
#pragma unroll
        for (int c = 0; c < kPacks; ++c) {
            xp[c] = xn[c];
            dp[c] = dn[c];
        }
        const float q = qn, m = mn;
        if constexpr (kHeld)
            ahead(r + step);
        auto weight = [&](int k) { return kHeld ? wv[kHeld ? k : 0] : shared[k * slot + threadIdx.x]; };
        auto hat = [&](int k) { return (to_f32(xp[k / kVec].v[k % kVec]) - m) * q; };
        float s[2] = {0.0f, 0.0f};
        // (past the row's end dy is 0, and with it all that is summed)
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const float xh = hat(k), up = to_f32(dp[k / kVec].v[k % kVec]), d = up * weight(k);
            if constexpr (kHeld) {
                dw[k] += up * xh;
                db[k] += up;
            } else {
                shared[(kPer + k) * slot + threadIdx.x] += up * xh;
                shared[(2 * kPer + k) * slot + threadIdx.x] += up;
            }
            s[0] += d;
            s[1] += d * xh;
        }
        group_sum<kGroup>(s, g, slots, turn);
        if (r >= rows)
            continue;
        const float a = s[0] * per * q, c1 = s[1] * per * q;
        T *out = dx + r * dxs;
#pragma unroll
        for (int c = 0; c < kPacks; ++c) {
            const int i = c * wide + at;
            Pack<T, kVec> o;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                const int k = c * kVec + e;
                const float d = to_f32(dp[c].v[e]) * weight(k);
                o.v[e] = from_f32<T>((q * d - a) - hat(k) * c1);
            }
            if (i < n)
                put<T, kVec>(out + i, o);
        }
    }
    if (!parts)
        return;
    float *mine = parts + (int64_t)blockIdx.x * 2 * n;
    if (g.count > 1) {
        if constexpr (kHeld) {
            if constexpr (kGroup > 0 && kGroup < 32) {  // groups of a warp first
#pragma unroll
                for (int o = kGroup; o < 32; o <<= 1) {
#pragma unroll
                    for (int k = 0; k < kPer; ++k) {
                        dw[k] += __shfl_xor_sync(~0u, dw[k], o);
                        db[k] += __shfl_xor_sync(~0u, db[k], o);
                    }
                }
            }
            const int team = kGroup && kGroup < 32 ? 32 : g.size, all = g.size * kPer;
            const bool speaks = threadIdx.x % team < g.size;
            for (int t = 0; t < (int)blockDim.x / team; ++t) {
                if ((int)threadIdx.x / team == t && speaks) {
#pragma unroll
                    for (int k = 0; k < kPer; ++k) {
                        const int i = k / kVec * wide + at + k % kVec;
                        shared[i] = (t ? shared[i] : 0.0f) + dw[k];
                        shared[all + i] = (t ? shared[all + i] : 0.0f) + db[k];
                    }
                }
                __syncthreads();
            }
            for (int i = threadIdx.x; i < n; i += blockDim.x) {
                mine[i] = shared[i];
                mine[n + i] = shared[all + i];
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int i = k / kVec * wide + at + k % kVec;
            if (i < n) {
                mine[i] = kHeld ? dw[kHeld ? k : 0] : shared[(kPer + k) * slot + threadIdx.x];
                mine[n + i] = kHeld ? db[kHeld ? k : 0] : shared[(2 * kPer + k) * slot + threadIdx.x];
            }
        }
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
        for (int i = threadIdx.x; i < n; i += kLongThreads)
            v += to_f32(xr[i]);
        const float m = long_sum(v, s) / n;
        v = 0.0f;
#pragma unroll 8
        for (int i = threadIdx.x; i < n; i += kLongThreads) {
            const float c = to_f32(xr[i]) - m;
            v += c * c;
        }
        const float q = 1.0f / sqrtf(long_sum(v, s) / n + eps);
#pragma unroll 8
        for (int i = threadIdx.x; i < n; i += kLongThreads)
            y[r * ys + i] = from_f32<T>((to_f32(xr[i]) - m) * q * param(w, ptype, i, 1.0f) + param(b, ptype, i, 0.0f));
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
        for (int i = threadIdx.x; i < n; i += kLongThreads) {
            const float d = to_f32(dr[i]) * param(w, ptype, i, 1.0f);
            a += d;
            c += d * (to_f32(xr[i]) - m) * q;
        }
        a = long_sum(a, s) / n;
        c = long_sum(c, s) / n;
#pragma unroll 8
        for (int i = threadIdx.x; i < n; i += kLongThreads) {
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

// The group, the block and the values a thread for rows of n values: 16 where
// 16 bytes hold eight of them, else 8.
struct Shape {
    int group, block, per;
    bool held;  // 128 registers a thread (85 in blocks of up to 768)
};
Shape shape_of(int n, bool sixteen)
{
    Shape s;
    s.per = sixteen ? 16 : 8;
    s.group = 2;
    while (s.group < 32 && s.group * s.per < n)
        s.group *= 2;
    if (s.group * s.per < n)
        s.group = (n + 32 * s.per - 1) / (32 * s.per) * 32;
    if (s.group > 1024) {
        s.per *= 2;
        s.group = (n + 32 * s.per - 1) / (32 * s.per) * 32;
    }
    s.block = s.group > kBlock ? s.group : kBlock / s.group * s.group;
    s.held = s.group <= (sixteen ? 512 : 768) && s.group * s.per <= 8192;
    return s;
}

// Blocks of a launch: one a SM (its registers are full), or what there is to do.
int blocks_of(int64_t rows, int n, bool sixteen)
{
    if (n > kLongest)
        return (int)(rows < 4 * kSms ? rows : 4 * kSms);
    const Shape s = shape_of(n, sixteen);
    const int64_t need = (rows + s.block / s.group - 1) / (s.block / s.group);
    return (int)(need < kSms ? need : kSms);
}

// Rows' parts of the column sums of long rows: blocks for every SM, eight rows each at least.
int long_parts(int64_t rows, int n)
{
    const int64_t slabs = (n + 31) / 32, want = (8 * kSms + slabs - 1) / slabs, most = (rows + 7) / 8;
    return (int)(want < most ? want : most);
}

int parts_of(int64_t rows, int n, bool sixteen)
{
    return n > kLongest ? long_parts(rows, n) : blocks_of(rows, n, sixteen);
}

// Rows that start on 16 bytes and hold whole packs of them.
bool packs(int64_t rows, int n, int e, const void *p, int64_t stride)
{
    return n % (16 / e) == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (rows <= 1 || stride * e % 16 == 0);
}

// Calls f with the values a thread, the threads a group (0: whole warps) and
// the threads a block at most as constants.
template <int kPer, class F>
void with_shape(const Shape &s, F f)
{
    using std::integral_constant;
#define AV_GROUP(g)          \
    if (s.group == g)        \
        return f(integral_constant<int, kPer>(), integral_constant<int, g>(), integral_constant<int, 512>());
    AV_GROUP(2) AV_GROUP(4) AV_GROUP(8) AV_GROUP(16) AV_GROUP(32)
#undef AV_GROUP
    if constexpr (kPer == 8) {
        if (s.per == 16)
            return f(integral_constant<int, 16>(), integral_constant<int, 0>(), integral_constant<int, 1024>());
        if (s.held && s.group > 512)
            return f(integral_constant<int, 8>(), integral_constant<int, 0>(), integral_constant<int, 768>());
    }
    if (s.held)
        return f(integral_constant<int, kPer>(), integral_constant<int, 0>(), integral_constant<int, 512>());
    f(integral_constant<int, kPer>(), integral_constant<int, 0>(), integral_constant<int, 1024>());
}

}  // namespace

// (of either shape: the larger)
int64_t norm_work_bytes(int64_t rows, int n)
{
    const int64_t a = parts_of(rows, n, true), b = parts_of(rows, n, false);
    return (a > b ? a : b) * 2 * n * 4;
}

cudaError_t launch_norm(int64_t rows, int n, int dtype, int param_dtype, float eps, const void *x, int64_t x_stride,
                        const void *weight, const void *bias, void *y, int64_t y_stride, float *mean, float *rstd,
                        cudaStream_t st)
{
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int kWide = 16 / sizeof(T);
        const bool wide = packs(rows, n, sizeof(T), x, x_stride) && packs(rows, n, sizeof(T), y, y_stride);
        const bool sixteen = wide && sizeof(T) == 2;
        const int blocks = blocks_of(rows, n, sixteen);
        if (n > kLongest) {
            norm_long_kernel<T><<<blocks, kLongThreads, 0, st>>>(rows, n, eps, (const T *)x, x_stride, weight, bias,
                                                                 param_dtype, (T *)y, y_stride, mean, rstd);
            return cudaGetLastError();
        }
        const Shape s = shape_of(n, sixteen);
        cudaError_t e = cudaSuccess;
        const int shared = s.held ? 0 : 2 * s.per * s.block * 4;
        auto run = [&](auto kernel) {
            if (shared > 48 * 1024)
                e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
            if (e == cudaSuccess)
                kernel<<<blocks, s.block, shared, st>>>(rows, n, s.group, eps, (const T *)x, x_stride, weight, bias,
                                                        param_dtype, (T *)y, y_stride, mean, rstd);
        };
        if (wide)
            with_shape<sizeof(T) == 2 ? 16 : 8>(s, [&](auto per, auto group, auto most) {
                run(norm_kernel<T, kWide, per.value, group.value, most.value>);
            });
        else
            with_shape<8>(s, [&](auto per, auto group, auto most) {
                run(norm_kernel<T, 1, per.value, group.value, most.value>);
            });
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
    const bool sixteen = wide && e_bytes == 2;
    const int count = parts_of(rows, n, sixteen);
    float *parts = (float *)work;
    cudaError_t e = cudaSuccess;
    if (rows > 0) {
        e = with_type(dtype, [&](auto t) {
            using T = decltype(t);
            constexpr int kWide = 16 / sizeof(T);
            const int blocks = blocks_of(rows, n, sixteen);
            if (n > kLongest) {
                norm_long_dx_kernel<T><<<blocks, kLongThreads, 0, st>>>(rows, n, (const T *)dy, dy_stride,
                                                                        (const T *)x, x_stride, weight, param_dtype,
                                                                        mean, rstd, (T *)dx, dx_stride);
                if (sums)
                    norm_long_columns_kernel<T><<<dim3((n + 31) / 32, count), 256, 0, st>>>(
                        rows, n, (const T *)dy, dy_stride, (const T *)x, x_stride, mean, rstd, parts);
                return cudaGetLastError();
            }
            const Shape s = shape_of(n, sixteen);
            cudaError_t bad = cudaSuccess;
            // parameters and running sums, or the groups' sums on their way together
            const int shared = s.held ? (s.block > s.group ? 2 * s.group * s.per * 4 : 0) : 3 * s.per * s.block * 4;
            auto run = [&](auto kernel) {
                if (shared > 48 * 1024)
                    bad = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, shared);
                if (bad == cudaSuccess)
                    kernel<<<blocks, s.block, shared, st>>>(rows, n, s.group, (const T *)dy, dy_stride, (const T *)x,
                                                            x_stride, weight, param_dtype, mean, rstd, (T *)dx,
                                                            dx_stride, sums ? parts : nullptr);
            };
            if (wide)
                with_shape<sizeof(T) == 2 ? 16 : 8>(s, [&](auto per, auto group, auto most) {
                    run(norm_grad_kernel<T, kWide, per.value, group.value, most.value>);
                });
            else
                with_shape<8>(s, [&](auto per, auto group, auto most) {
                    run(norm_grad_kernel<T, 1, per.value, group.value, most.value>);
                });
            return bad != cudaSuccess ? bad : cudaGetLastError();
        });
        if (e != cudaSuccess)
            return e;
    }
    if (sums)
        norm_columns_kernel<<<dim3((n + kColumns - 1) / kColumns, 2), 256, 0, st>>>(count, n, parts, param_dtype,
                                                                                   dweight, dbias);
    return cudaGetLastError();
}

}  // namespace av
