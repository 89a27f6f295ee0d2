// k_scan.cu -- the gated linear recurrence and its gradient.
//   forward   a = sigmoid(g), h_t = a k_t h_{t-1} + (1 - a) v_t
//   backward  l_t = dh_t + a_{t+1} k_{t+1} l_{t+1}; dv = (1 - a) l; dg = l (k h_{t-1} - v) a (1 - a)
//
// Steps are affine maps h -> A h + H, and maps compose: a run of steps is one
// map whatever its length.  A block takes 32 lanes of channels and a chunk of
// steps, each of its eight warps a run of them.  The run is read once into
// registers, its map goes to shared memory, and with the state before the run
// (the chunk's, carried through the maps of the runs before) the steps are
// taken from registers.  So both directions read and write their arrays once:
// 3 and 5 values a step and channel.  The backward pass makes the states again
// from the one kept at each chunk's start (4 bytes a chunk and channel), so it
// neither reads h nor suffers its rounding.  Bound by memory.
//
// Where channels alone fill the GPU, a block walks its channels' chunks in
// order.  Where they do not, every chunk is a block: it publishes its map and
// takes the state from the maps of the chunks before it in its group of 32 and
// the state at the group's start, in that fixed order, whoever is ready first.
// Blocks draw their places from a counter, so what one waits for has begun.
//
// A step that begins an episode forgets the state even where it is NaN: in a
// map this is A = -0, whose sign survives composition.
#include <stdlib.h>

#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kWarps = 8;        // runs of a chunk
constexpr int kThreads = 32 * kWarps;
constexpr int kLongRun = 16, kShortRun = 4;  // steps of a run
constexpr int kGroup = 32;       // chunks that share a start
constexpr int64_t kEnough = 912; // blocks of channels that fill the GPU without chunks of their own

// min(a, 1 - a) of a = sigmoid(g), its sign telling which: negative where it is
// a itself.  One register holds both a and 1 - a without cancellation.
__device__ __forceinline__ float squash(float g)
{
    const float e = __expf(-fabsf(g));
    return copysignf(__fdividef(e, 1.0f + e), g);
}
__device__ __forceinline__ bool marked(float v) { return __float_as_int(v) < 0; }
__device__ __forceinline__ float gate_of(float q) { return marked(q) ? fabsf(q) : 1.0f - q; }
__device__ __forceinline__ float rest_of(float q) { return marked(q) ? 1.0f + q : q; }

// A run's registers, to be read anew: what was computed from them is not kept.
template <class V, int kRun, int kVec>
__device__ __forceinline__ void renew(V (&r)[kRun], float (&q)[kRun][kVec])
{
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
        if constexpr (sizeof(V) == 4)
            asm volatile("" : "+r"(*reinterpret_cast<uint32_t *>(&r[k])));
        else
            asm volatile("" : "+h"(*reinterpret_cast<uint16_t *>(&r[k])));
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            asm volatile("" : "+f"(q[k][v]));
    }
}

// The map's value at h; A = -0 forgets h.
__device__ __forceinline__ float apply(float A, float H, float h) { return marked(A) ? H : fmaf(A, h, H); }
// The factor of first A1, then A2.
__device__ __forceinline__ float then(float A1, float A2) { return marked(A1) || marked(A2) ? -0.0f : A1 * A2; }

// Where the arrays of a call lie.
struct Args {
    int64_t T, B, D;
    const void *gate, *value, *dh;
    int64_t gt, gb, vt, vb, ht, hb;  // ht, hb: of dh backward, of h forward
    const uint8_t *reset;
    int64_t rt, rb;
    void *h;                // forward
    const float *first;     // h0 forward, dlast backward: the state that enters, or NULL
    float *last;            // h_last forward, dh0 backward: the state that leaves, or NULL
    float *states;          // [chunk][B D]: written forward (or NULL), read backward
    void *dgate, *dvalue;   // backward
    int64_t dgt, dgb, dvt, dvb;
    int64_t slabs, chunks;  // blocks of channels, chunks of steps
    int *ticket;            // NULL: a block walks all chunks
    int *ready, *group_ready;       // [slab][chunk], [slab][group]
    float2 *maps;                   // [slab][chunk][channel]
    float *group_state;             // [slab][group][channel]
    int64_t limit_ns;
};

__device__ __forceinline__ int load_flag(const int *p)
{
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store_flag(int *p)
{
    asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(1) : "memory");
}
__device__ __forceinline__ int64_t now_ns()
{
    int64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Waits for a flag; false when the limit passes first (a negative one: at once).
__device__ __noinline__ bool wait_flag(const int *p, int64_t limit_ns)
{
    if (limit_ns < 0)
        return false;
    int64_t began = 0;
    for (int spins = 0; load_flag(p) == 0; ++spins) {
        if ((spins & 255) == 255) {
            const int64_t t = now_ns();
            if (!began)
                began = t;
            else if (t - began > limit_ns)
                return false;
        }
    }
    return true;
}

// kVec neighbouring values: one load.
template <class T, int kVec>
struct Few {
    T v[kVec];
};
template <class T, int kVec>
__device__ __forceinline__ Few<T, kVec> fetch(const T *p)
{
    Few<T, kVec> r;
    if constexpr (kVec == 1)
        r.v[0] = *p;
    else
        *reinterpret_cast<uint32_t *>(&r) = *reinterpret_cast<const uint32_t *>(p);
    return r;
}
template <class T, int kVec>
__device__ __forceinline__ void put(T *p, const Few<T, kVec> &r)
{
    if constexpr (kVec == 1)
        *p = r.v[0];
    else
        *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(&r);
}

// The state at the start of the chunk at `place` of its chain (forward: the
// chunk; backward: chunks from the end), from the chunks before it, and the
// chunk's own map for those after.  total: the chunk's map, by warp 0's lanes;
// scratch: a map a warp and channel.  Returns a value for this lane's channels.
template <int kVec>
__device__ void chained(const Args &a, int64_t slab, int64_t place, const float (&A)[kVec], const float (&H)[kVec],
                        float2 (*scratch)[32 * kVec], float (&state)[kVec])
{
    constexpr int kSlab = 32 * kVec;
    __shared__ float start[kSlab];
    __shared__ int late;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t group = place / kGroup, groups = (a.chunks + kGroup - 1) / kGroup;
    const int before = (int)(place % kGroup);
    float2 *maps = a.maps + slab * a.chunks * kSlab;
    if (threadIdx.x == 0)
        late = 0;
    if (warp == 0) {
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            __stcg(&maps[place * kSlab + lane * kVec + v], make_float2(A[v], H[v]));
        __threadfence();
        __syncwarp();
        if (lane == 0)
            store_flag(a.ready + slab * a.chunks + place);
    }
    __syncthreads();
    // four chunks of the group a warp, composed in order
    const int c0 = warp * 4, c1 = before < c0 + 4 ? before : c0 + 4;
    const int64_t base = group * kGroup;
    if (c0 + lane < c1 && !wait_flag(a.ready + slab * a.chunks + base + c0 + lane, a.limit_ns))
        late = 1;
    __syncwarp();
    float2 m[4][kVec];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            m[c][v] = c0 + c < c1 ? __ldcg(&maps[(base + c0 + c) * kSlab + lane * kVec + v]) : make_float2(1.0f, 0.0f);
    }
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
        float2 t = m[0][v];
#pragma unroll
        for (int c = 1; c < 4; ++c) {
            t.y = apply(m[c][v].x, m[c][v].y, t.y);
            t.x = then(t.x, m[c][v].x);
        }
        scratch[warp][lane * kVec + v] = t;
    }
    if (warp == 0) {
        if (group > 0) {
            if (lane == 0 && !wait_flag(a.group_ready + slab * groups + group - 1, a.limit_ns))
                late = 1;
            __syncwarp();
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                start[lane * kVec + v] = __ldcg(&a.group_state[(slab * groups + group - 1) * kSlab + lane * kVec + v]);
        } else {
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                const int64_t c = slab * kSlab + lane * kVec + v;
                start[lane * kVec + v] = a.first && c < a.B * a.D ? a.first[c] : 0.0f;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kVec; ++v) {
        float s = start[lane * kVec + v];
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
            s = apply(scratch[w][lane * kVec + v].x, scratch[w][lane * kVec + v].y, s);
        state[v] = late ? __int_as_float(0x7fffffff) : s;
    }
    if (warp == 0 && before == kGroup - 1) {
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            __stcg(&a.group_state[(slab * groups + group) * kSlab + lane * kVec + v], apply(A[v], H[v], state[v]));
        __threadfence();
        __syncwarp();
        if (lane == 0)
            store_flag(a.group_ready + slab * groups + group);
    }
}

// Bits of the run's steps that begin an episode, of this lane's sequence.
template <int kRun>
__device__ __forceinline__ uint32_t resets_of(const Args &a, int64_t t0, int64_t b, bool valid, bool same)
{
    if (!a.reset)
        return 0;
    uint32_t mask = 0;
    if (same) {  // the whole warp reads one sequence: a step a lane
        const int lane = threadIdx.x & 31;
        const bool hit = lane < kRun && t0 + lane < a.T && a.reset[(t0 + lane) * a.rt + b * a.rb] != 0;
        return __ballot_sync(~0u, hit);
    }
#pragma unroll
    for (int k = 0; k < kRun; ++k)
        if (valid && t0 + k < a.T && a.reset[(t0 + k) * a.rt + b * a.rb] != 0)
            mask |= 1u << k;
    return mask;
}

template <class T, int kVec, int kRun>
__global__ __launch_bounds__(kThreads, 2) void scan_kernel(const Args a)
{
    constexpr int kSlab = 32 * kVec, kChunk = kRun * kWarps;
    __shared__ float2 runs[kWarps][kSlab], others[kWarps][kSlab];
    __shared__ float carry[kSlab];
    __shared__ int drawn;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t slab = blockIdx.x, chunk = 0, end = a.chunks;
    if (a.ticket) {
        if (threadIdx.x == 0)
            drawn = atomicAdd(a.ticket, 1);
        __syncthreads();
        chunk = (unsigned)drawn / a.slabs;
        slab = (unsigned)drawn % a.slabs;
        end = chunk + 1;
    }
    const int64_t n = a.B * a.D, c = slab * kSlab + lane * kVec;
    const bool valid = c < n;
    const int64_t b = valid ? c / a.D : (n - 1) / a.D, d = valid ? c % a.D : 0;
    const bool same = __all_sync(~0u, b == __shfl_sync(~0u, b, 0));
    const T *gate = (const T *)a.gate + b * a.gb + d, *value = (const T *)a.value + b * a.vb + d;
    T *h = (T *)a.h + b * a.hb + d;
    if (!a.ticket && warp == 0) {
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            carry[lane * kVec + v] = valid && a.first ? a.first[c + v] : 0.0f;
    }
    for (; chunk < end; ++chunk) {
        const int64_t t0 = chunk * kChunk + warp * kRun;
        Few<T, kVec> gp[kRun], vp[kRun];
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            if (valid && t0 + k < a.T) {
                gp[k] = fetch<T, kVec>(gate + (t0 + k) * a.gt);
                vp[k] = fetch<T, kVec>(value + (t0 + k) * a.vt);
            } else {  // a step that changes nothing
#pragma unroll
                for (int v = 0; v < kVec; ++v) {
                    gp[k].v[v] = from_f32<T>(INFINITY);
                    vp[k].v[v] = from_f32<T>(0.0f);
                }
            }
        }
        const uint32_t resets = resets_of<kRun>(a, t0, b, valid, same);
        float q[kRun][kVec], A[kVec], H[kVec];
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
            A[v] = 1.0f;
            H[v] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const bool keep = !(resets >> k & 1);
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                q[k][v] = squash(to_f32(gp[k].v[v]));
                const float g = gate_of(q[k][v]);
                H[v] = (keep ? g * H[v] : 0.0f) + rest_of(q[k][v]) * to_f32(vp[k].v[v]);
                A[v] *= g;
            }
        }
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
            if (resets)
                A[v] = -0.0f;
            runs[warp][lane * kVec + v] = make_float2(A[v], H[v]);
        }
        __syncthreads();
        renew(vp, q);
        float s[kVec];
        if (a.ticket) {
            float TA[kVec], TH[kVec];
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                TA[v] = 1.0f;
                TH[v] = 0.0f;
                if (warp == 0) {
                    for (int w = 0; w < kWarps; ++w) {
                        const float2 m = runs[w][lane * kVec + v];
                        TH[v] = apply(m.x, m.y, TH[v]);
                        TA[v] = then(TA[v], m.x);
                    }
                }
            }
            chained<kVec>(a, slab, chunk, TA, TH, others, s);
        } else {
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                s[v] = carry[lane * kVec + v];
        }
        if (a.states && warp == 0 && valid) {
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                a.states[chunk * n + c + v] = s[v];
        }
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            for (int w = 0; w < warp; ++w)
                s[v] = apply(runs[w][lane * kVec + v].x, runs[w][lane * kVec + v].y, s[v]);
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const bool keep = !(resets >> k & 1);
            Few<T, kVec> o;
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                s[v] = (keep ? gate_of(q[k][v]) * s[v] : 0.0f) + rest_of(q[k][v]) * to_f32(vp[k].v[v]);
                o.v[v] = from_f32<T>(s[v]);
            }
            if (valid && t0 + k < a.T)
                put<T, kVec>(h + (t0 + k) * a.ht, o);
        }
        if (warp == kWarps - 1 && valid && chunk == a.chunks - 1 && a.last) {
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                a.last[c + v] = s[v];
        }
        if (!a.ticket) {
            __syncthreads();  // (all have read the carry and the runs)
            if (warp == kWarps - 1) {
#pragma unroll
                for (int v = 0; v < kVec; ++v)
                    carry[lane * kVec + v] = s[v];
            }
            // (read next behind the barrier after the next runs)
        }
    }
}

// Backward: chunks from the last to the first.  What flows to before step t is
// m_t = a_t k_t l_t, l_t = dh_t + m_{t+1}: a run's map of it has the forward
// map's factor.
template <class T, int kVec, int kRun>
__global__ __launch_bounds__(kThreads, 2) void scan_grad_kernel(const Args a)
{
    constexpr int kSlab = 32 * kVec, kChunk = kRun * kWarps;
    __shared__ float2 runs[kWarps][kSlab], flows[kWarps][kSlab], others[kWarps][kSlab];
    __shared__ float carry[kSlab];
    __shared__ int drawn;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t slab = blockIdx.x, place = 0, end = a.chunks;
    if (a.ticket) {
        if (threadIdx.x == 0)
            drawn = atomicAdd(a.ticket, 1);
        __syncthreads();
        place = (unsigned)drawn / a.slabs;
        slab = (unsigned)drawn % a.slabs;
        end = place + 1;
    }
    const int64_t n = a.B * a.D, c = slab * kSlab + lane * kVec;
    const bool valid = c < n;
    const int64_t b = valid ? c / a.D : (n - 1) / a.D, d = valid ? c % a.D : 0;
    const bool same = __all_sync(~0u, b == __shfl_sync(~0u, b, 0));
    const T *gate = (const T *)a.gate + b * a.gb + d, *value = (const T *)a.value + b * a.vb + d;
    const T *dh = (const T *)a.dh + b * a.hb + d;
    T *dgate = (T *)a.dgate + b * a.dgb + d, *dvalue = (T *)a.dvalue + b * a.dvb + d;
    if (!a.ticket && warp == 0) {
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            carry[lane * kVec + v] = valid && a.first ? a.first[c + v] : 0.0f;
    }
    for (; place < end; ++place) {
        const int64_t chunk = a.chunks - 1 - place, t0 = chunk * kChunk + warp * kRun;
        Few<T, kVec> gp[kRun], vp[kRun], dp[kRun];
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            if (valid && t0 + k < a.T) {
                gp[k] = fetch<T, kVec>(gate + (t0 + k) * a.gt);
                vp[k] = fetch<T, kVec>(value + (t0 + k) * a.vt);
                dp[k] = fetch<T, kVec>(dh + (t0 + k) * a.ht);
            } else {
#pragma unroll
                for (int v = 0; v < kVec; ++v) {
                    gp[k].v[v] = from_f32<T>(INFINITY);
                    vp[k].v[v] = dp[k].v[v] = from_f32<T>(0.0f);
                }
            }
        }
        float s[kVec];
#pragma unroll
        for (int v = 0; v < kVec; ++v)
            s[v] = valid ? a.states[chunk * n + c + v] : 0.0f;
        const uint32_t resets = resets_of<kRun>(a, t0, b, valid, same);
        float q[kRun][kVec], A[kVec], H[kVec], Q[kVec];
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
            A[v] = 1.0f;
            H[v] = Q[v] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const bool keep = !(resets >> k & 1);
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                q[k][v] = squash(to_f32(gp[k].v[v]));
                const float g = gate_of(q[k][v]);
                H[v] = (keep ? g * H[v] : 0.0f) + rest_of(q[k][v]) * to_f32(vp[k].v[v]);
                A[v] *= g;
            }
        }
#pragma unroll
        for (int k = kRun - 1; k >= 0; --k) {
            const bool keep = !(resets >> k & 1);
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                Q[v] = keep ? gate_of(q[k][v]) * (to_f32(dp[k].v[v]) + Q[v]) : 0.0f;
        }
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
            if (resets)
                A[v] = -0.0f;
            runs[warp][lane * kVec + v] = make_float2(A[v], H[v]);
            flows[warp][lane * kVec + v] = make_float2(A[v], Q[v]);
        }
        __syncthreads();
        renew(vp, q);
        renew(dp, q);
        float m[kVec];
        if (a.ticket) {
            float TA[kVec], TQ[kVec];
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                TA[v] = 1.0f;
                TQ[v] = 0.0f;
                if (warp == 0) {
                    for (int w = kWarps - 1; w >= 0; --w) {
                        const float2 f = flows[w][lane * kVec + v];
                        TQ[v] = apply(f.x, f.y, TQ[v]);
                        TA[v] = then(TA[v], f.x);
                    }
                }
            }
            chained<kVec>(a, slab, place, TA, TQ, others, m);
        } else {
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                m[v] = carry[lane * kVec + v];
        }
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
            for (int w = 0; w < warp; ++w)
                s[v] = apply(runs[w][lane * kVec + v].x, runs[w][lane * kVec + v].y, s[v]);
            for (int w = kWarps - 1; w > warp; --w)
                m[v] = apply(flows[w][lane * kVec + v].x, flows[w][lane * kVec + v].y, m[v]);
        }
        renew(vp, q);
        float u[kRun][kVec];  // k h_{t-1} - v_t
#pragma unroll
        for (int k = 0; k < kRun; ++k) {
            const bool keep = !(resets >> k & 1);
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                const float x = to_f32(vp[k].v[v]), held = keep ? s[v] : 0.0f;
                u[k][v] = held - x;
                s[v] = (keep ? gate_of(q[k][v]) * s[v] : 0.0f) + rest_of(q[k][v]) * x;
            }
        }
        renew(dp, q);
#pragma unroll
        for (int k = kRun - 1; k >= 0; --k) {
            const bool keep = !(resets >> k & 1);
            Few<T, kVec> og, ov;
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                const float g = gate_of(q[k][v]), z = rest_of(q[k][v]), l = to_f32(dp[k].v[v]) + m[v];
                ov.v[v] = from_f32<T>(z * l);
                og.v[v] = from_f32<T>(l * u[k][v] * (g * z));
                m[v] = keep ? g * l : 0.0f;
            }
            if (valid && t0 + k < a.T) {
                put<T, kVec>(dvalue + (t0 + k) * a.dvt, ov);
                put<T, kVec>(dgate + (t0 + k) * a.dgt, og);
            }
        }
        if (warp == 0 && valid && chunk == 0 && a.last) {
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                a.last[c + v] = m[v];
        }
        if (!a.ticket) {
            __syncthreads();
            if (warp == 0) {
#pragma unroll
                for (int v = 0; v < kVec; ++v)
                    carry[lane * kVec + v] = m[v];
            }
        }
    }
}

// One step: every value once, kVec at a time.
template <class T, int kVec>
__global__ __launch_bounds__(256) void step_kernel(const Args a)
{
    const int64_t n = a.B * a.D, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * kVec;
    if (c >= n)
        return;
    const int64_t b = c / a.D, d = c % a.D;
    const bool keep = !a.reset || a.reset[b * a.rb] == 0;
    T g[kVec], v[kVec];
    float s[kVec] = {};
    const T *gp = (const T *)a.gate + b * a.gb + d, *vp = (const T *)a.value + b * a.vb + d;
    if constexpr (kVec > 1) {
        *reinterpret_cast<uint4 *>(g) = *reinterpret_cast<const uint4 *>(gp);
        *reinterpret_cast<uint4 *>(v) = *reinterpret_cast<const uint4 *>(vp);
        if (a.first) {
#pragma unroll
            for (int k = 0; k < kVec; k += 4)
                *reinterpret_cast<float4 *>(s + k) = *reinterpret_cast<const float4 *>(a.first + c + k);
        }
    } else {
        g[0] = *gp;
        v[0] = *vp;
        if (a.first)
            s[0] = a.first[c];
    }
    T o[kVec];
    float next[kVec];
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
        const float q = squash(to_f32(g[k]));
        next[k] = (keep ? gate_of(q) * s[k] : 0.0f) + rest_of(q) * to_f32(v[k]);
        o[k] = from_f32<T>(next[k]);
    }
    T *hp = (T *)a.h + b * a.hb + d;
    if constexpr (kVec > 1) {
        *reinterpret_cast<uint4 *>(hp) = *reinterpret_cast<const uint4 *>(o);
#pragma unroll
        for (int k = 0; k < kVec; k += 4) {
            if (a.states)
                *reinterpret_cast<float4 *>(a.states + c + k) = *reinterpret_cast<const float4 *>(s + k);
            if (a.last)
                *reinterpret_cast<float4 *>(a.last + c + k) = *reinterpret_cast<const float4 *>(next + k);
        }
    } else {
        *hp = o[0];
        if (a.states)
            a.states[c] = s[0];
        if (a.last)
            a.last[c] = next[0];
    }
}

// ------------------------------------------------------------ host

// Steps a run: short sequences leave no warp without one.
int run_of(int64_t T) { return T <= kShortRun * kWarps ? kShortRun : kLongRun; }

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Channels of a lane: a 32-bit word of them, where both an element's
// neighbour is of the same sequence and all arrays keep pairs together.
bool pairs(int64_t D, int dtype, const void *p, int64_t t, int64_t b)
{
    return dtype != AV_F32 && D % 2 == 0 && (reinterpret_cast<uintptr_t>(p) & 3) == 0 && t % 2 == 0 && b % 2 == 0;
}

// Blocks of channels are counted with one channel a lane: an upper bound of
// those with two, so a workspace fits either.
struct Plan {
    int64_t chunks, groups, slabs;
    bool chained;
};
Plan plan_of(int64_t T, int64_t n, int wide)
{
    Plan p;
    p.chunks = up(T, run_of(T) * kWarps);
    p.groups = up(p.chunks, kGroup);
    p.slabs = up(n, 32 * wide);
    p.chained = p.chunks > 1 && p.slabs < kEnough;
    return p;
}

int64_t flag_bytes(const Plan &p) { return up((1 + p.slabs * (p.chunks + p.groups)) * 4, 256) * 256; }

int64_t plan_bytes(const Plan &p, int wide)
{
    if (!p.chained)
        return 0;
    return flag_bytes(p) + p.slabs * 32 * wide * (p.chunks * 8 + p.groups * 4);
}

// Lays the workspace out; clears the counter and the flags.
cudaError_t arrange(Args &a, const Plan &p, int wide, void *work, cudaStream_t st)
{
    a.slabs = p.slabs;
    a.chunks = p.chunks;
    if (!p.chained)
        return cudaSuccess;
    a.ticket = (int *)work;
    a.ready = a.ticket + 1;
    a.group_ready = a.ready + p.slabs * p.chunks;
    a.maps = (float2 *)((char *)work + flag_bytes(p));
    a.group_state = (float *)(a.maps + p.slabs * p.chunks * 32 * wide);
    a.limit_ns = 4000000000ll;
    if (const char *ms = getenv("AV_SCAN_WAIT_MS"))  // for tests of the limit
        a.limit_ns = atoll(ms) * 1000000;
    return cudaMemsetAsync(work, 0, flag_bytes(p), st);
}

}  // namespace

void scan_sizes(int64_t T, int64_t B, int64_t D, int dtype, int64_t *states, int64_t *work)
{
    const int64_t one = plan_bytes(plan_of(T, B * D, 1), 1);
    const int64_t two = dtype == AV_F32 ? 0 : plan_bytes(plan_of(T, B * D, 2), 2);
    *states = up(T, run_of(T) * kWarps) * B * D;
    *work = one > two ? one : two;
}

cudaError_t launch_scan(int64_t T, int64_t B, int64_t D, int dtype, Seq gate, Seq value, Seq reset, const float *h0,
                        SeqOut h, float *h_last, float *states, void *work, cudaStream_t st)
{
    Args a{};
    a.T = T, a.B = B, a.D = D;
    a.gate = gate.p, a.gt = gate.t, a.gb = gate.b;
    a.value = value.p, a.vt = value.t, a.vb = value.b;
    a.reset = (const uint8_t *)reset.p, a.rt = reset.t, a.rb = reset.b;
    a.h = h.p, a.ht = h.t, a.hb = h.b;
    a.first = h0, a.last = h_last, a.states = states;
    const int64_t n = B * D;
    if (T == 1) {
        with_type(dtype, [&](auto v) {
            using E = decltype(v);
            constexpr int kWide = 16 / sizeof(E);
            auto whole = [&](const void *p, int64_t b, int64_t e) {
                return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && b * e % 16 == 0;
            };
            if (D % kWide == 0 && whole(gate.p, gate.b, sizeof(E)) && whole(value.p, value.b, sizeof(E)) &&
                whole(h.p, h.b, sizeof(E)) && whole(h0, 0, 4) && whole(h_last, 0, 4) && whole(states, 0, 4))
                step_kernel<E, kWide><<<(unsigned)up(n / kWide, 256), 256, 0, st>>>(a);
            else
                step_kernel<E, 1><<<(unsigned)up(n, 256), 256, 0, st>>>(a);
        });
        return cudaGetLastError();
    }
    const int wide = pairs(D, dtype, gate.p, gate.t, gate.b) && pairs(D, dtype, value.p, value.t, value.b) &&
                             pairs(D, dtype, h.p, h.t, h.b)
                         ? 2
                         : 1;
    const Plan p = plan_of(T, n, wide);
    const cudaError_t e = arrange(a, p, wide, work, st);
    if (e != cudaSuccess)
        return e;
    const unsigned grid = (unsigned)(p.chained ? p.slabs * p.chunks : p.slabs);
    with_type(dtype, [&](auto v) {
        using E = decltype(v);
        const bool brief = run_of(T) == kShortRun;
        if constexpr (sizeof(E) == 2) {
            if (wide == 2) {
                if (brief)
                    scan_kernel<E, 2, kShortRun><<<grid, kThreads, 0, st>>>(a);
                else
                    scan_kernel<E, 2, kLongRun><<<grid, kThreads, 0, st>>>(a);
                return;
            }
        }
        if (brief)
            scan_kernel<E, 1, kShortRun><<<grid, kThreads, 0, st>>>(a);
        else
            scan_kernel<E, 1, kLongRun><<<grid, kThreads, 0, st>>>(a);
    });
    return cudaGetLastError();
}

cudaError_t launch_scan_grad(int64_t T, int64_t B, int64_t D, int dtype, Seq dh, Seq gate, Seq value, Seq reset,
                             const float *states, const float *dlast, SeqOut dgate, SeqOut dvalue, float *dh0,
                             void *work, cudaStream_t st)
{
    Args a{};
    a.T = T, a.B = B, a.D = D;
    a.gate = gate.p, a.gt = gate.t, a.gb = gate.b;
    a.value = value.p, a.vt = value.t, a.vb = value.b;
    a.dh = dh.p, a.ht = dh.t, a.hb = dh.b;
    a.reset = (const uint8_t *)reset.p, a.rt = reset.t, a.rb = reset.b;
    a.first = dlast, a.last = dh0, a.states = const_cast<float *>(states);
    a.dgate = dgate.p, a.dgt = dgate.t, a.dgb = dgate.b;
    a.dvalue = dvalue.p, a.dvt = dvalue.t, a.dvb = dvalue.b;
    const int wide = pairs(D, dtype, gate.p, gate.t, gate.b) && pairs(D, dtype, value.p, value.t, value.b) &&
                             pairs(D, dtype, dh.p, dh.t, dh.b) && pairs(D, dtype, dgate.p, dgate.t, dgate.b) &&
                             pairs(D, dtype, dvalue.p, dvalue.t, dvalue.b)
                         ? 2
                         : 1;
    const Plan p = plan_of(T, B * D, wide);
    const cudaError_t e = arrange(a, p, wide, work, st);
    if (e != cudaSuccess)
        return e;
    const unsigned grid = (unsigned)(p.chained ? p.slabs * p.chunks : p.slabs);
    with_type(dtype, [&](auto v) {
        using E = decltype(v);
        const bool brief = run_of(T) == kShortRun;
        if constexpr (sizeof(E) == 2) {
            if (wide == 2) {
                if (brief)
                    scan_grad_kernel<E, 2, kShortRun><<<grid, kThreads, 0, st>>>(a);
                else
                    scan_grad_kernel<E, 2, kLongRun><<<grid, kThreads, 0, st>>>(a);
                return;
            }
        }
        if (brief)
            scan_grad_kernel<E, 1, kShortRun><<<grid, kThreads, 0, st>>>(a);
        else
            scan_grad_kernel<E, 1, kLongRun><<<grid, kThreads, 0, st>>>(a);
    });
    return cudaGetLastError();
}

}  // namespace av
