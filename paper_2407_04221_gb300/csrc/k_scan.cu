// k_scan.cu -- the gated linear recurrence and its gradient.
//   forward   a = sigmoid(g), h_t = a k_t h_{t-1} + (1 - a) v_t
//   backward  l_t = dh_t + a_{t+1} k_{t+1} l_{t+1}; dv = (1 - a) l; dg = l (k h_{t-1} - v) a (1 - a)
//
// Steps are affine maps h -> A h + H, and maps compose: a run of steps is one
// map whatever its length.  A block takes 64 channels and chunks of 128 steps
// (64 of 32-bit values, 32 or 64 of shorter sequences).  A warp takes eight of the channels: its
// lanes are four pairs of them by eight runs of 16 steps, so that runs are
// joined by shuffles and no warp waits for another.  Chunks come to shared
// memory by asynchronous copies, the next ones under way during this one, and
// results leave from the places of the inputs they came from; eight channels
// of a step are 16 bytes, whose place in the row turns with the run, so that
// lanes of different runs read different banks.  Both directions read and
// write their arrays once: 3 and 5 values a step and channel.  The backward
// pass makes the states again from the one kept at each chunk's start (4 bytes
// a chunk and channel), so it neither reads h nor suffers its rounding.  Bound
// by memory, and for 16-bit values nearly by issue: some 20 instructions a
// value forward.
//
// Where channels alone fill the GPU, a block walks its channels' chunks in
// order.  Where they do not, blocks take chunks as they come: a warp publishes
// its chunk's map and takes its state from the maps of the chunks before it in
// its group of 32 and the state at the group's start, in that fixed order,
// whoever is ready first.  Places are drawn from a counter, so what a chunk
// waits for was drawn before it.
//
// A step that begins an episode forgets the state even where it is NaN: in a
// map this is a factor with its sign bit set, which survives composition.
#include <stdlib.h>

#include <type_traits>

#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kRuns = 8;         // runs of a chunk, a quarter of a warp's lanes each
constexpr int kLongRun = 16;     // steps of a run at most
constexpr int kSlab = 64;        // channels of a block, eight a warp, two a lane
constexpr int kGroup = 32;       // chunks that share a start
constexpr int kSms = 152;

__device__ __forceinline__ float exp2_fast(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// a = sigmoid(g) and z = 1 - a without cancellation: e = exp(-g), 1 / (1 + e)
// and e / (1 + e).  Below g = -80 the gate stays at 2e-35.
__device__ __forceinline__ void gates_of(float2 g, float2 &a, float2 &z)
{
    float2 e = mul2(g, make_float2(-1.4426950408889634f, -1.4426950408889634f));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(e.x) : "f"(e.x), "f"(115.5f));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(e.y) : "f"(e.y), "f"(115.5f));
    e.x = exp2_fast(e.x);
    e.y = exp2_fast(e.y);
    const float2 d = add2(e, make_float2(1.0f, 1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.x) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.y) : "f"(d.y));
    z = mul2(e, a);
}
__device__ __forceinline__ bool marked(float v) { return __float_as_int(v) < 0; }
// The map's value at h; a marked factor forgets h.
__device__ __forceinline__ float apply(float A, float H, float h) { return marked(A) ? H : fmaf(A, h, H); }
// The factor of first A1, then A2.
__device__ __forceinline__ float then(float A1, float A2) { return marked(A1) || marked(A2) ? -0.0f : A1 * A2; }

struct Map2 {  // maps of a lane's two channels
    float A[2], H[2];
};
// First p, then q.
__device__ __forceinline__ Map2 then2(const Map2 &p, const Map2 &q)
{
    return {{then(p.A[0], q.A[0]), then(p.A[1], q.A[1])}, {apply(q.A[0], q.H[0], p.H[0]), apply(q.A[1], q.H[1], p.H[1])}};
}
__device__ __forceinline__ Map2 identity() { return {{1.0f, 1.0f}, {0.0f, 0.0f}}; }

// The maps of the runs up to and with each, runs in order (kBack: from the
// last); lanes of one pair of channels are four apart.
template <bool kBack>
__device__ __forceinline__ Map2 joined(Map2 m)
{
    const int run = (threadIdx.x & 31) >> 2;
#pragma unroll
    for (int o = 1; o < kRuns; o <<= 1) {
        Map2 before;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            before.A[v] = kBack ? __shfl_down_sync(~0u, m.A[v], 4 * o) : __shfl_up_sync(~0u, m.A[v], 4 * o);
            before.H[v] = kBack ? __shfl_down_sync(~0u, m.H[v], 4 * o) : __shfl_up_sync(~0u, m.H[v], 4 * o);
        }
        if (kBack ? run + o < kRuns : run >= o)
            m = then2(before, m);
    }
    return m;
}

// What is before each run, given what is joined: nothing before the first.
template <bool kBack>
__device__ __forceinline__ Map2 before_each(const Map2 &m)
{
    const int run = (threadIdx.x & 31) >> 2;
    Map2 b;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        b.A[v] = kBack ? __shfl_down_sync(~0u, m.A[v], 4) : __shfl_up_sync(~0u, m.A[v], 4);
        b.H[v] = kBack ? __shfl_down_sync(~0u, m.H[v], 4) : __shfl_up_sync(~0u, m.H[v], 4);
    }
    return (kBack ? run == kRuns - 1 : run == 0) ? identity() : b;
}

// The map of all runs, in every lane.
template <bool kBack>
__device__ __forceinline__ Map2 whole(const Map2 &m)
{
    const int from = (kBack ? 0 : 28) + (threadIdx.x & 3);
    Map2 t;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        t.A[v] = __shfl_sync(~0u, m.A[v], from);
        t.H[v] = __shfl_sync(~0u, m.H[v], from);
    }
    return t;
}

// Where the arrays of a call lie.
struct Args {
    int64_t T, B, D;
    const void *in[3];          // gate, value, dh
    int64_t it[3], ib[3];
    const uint8_t *reset;
    int64_t rt, rb;
    void *out[2];               // h, or dgate and dvalue
    int64_t ot[2], ob[2];
    const float *first;         // h0 forward, dlast backward: the state that enters, or NULL
    float *last;                // h_last forward, dh0 backward: the state that leaves, or NULL
    float *states;              // [chunk][B D]: written forward (or NULL), read backward
    uint32_t slabs, chunks;     // blocks of channels, chunks of steps
    bool flat;                  // sequences lie side by side: channels are numbered through
    int in_bytes, out_bytes;    // of a copy: 16, 4, or 0 where values are copied one by one
    int *ticket;                // NULL: a block walks all chunks
    int *ready, *group_ready;   // [slab][warp][chunk], [slab][warp][group]
    Map2 *maps;                 // [slab][warp][chunk][4]
    float2 *group_state;        // [slab][warp][group][4]
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

// What a block does next: chunk `place` chunks after its chain's first
// (backward: from the end) of a slab of channels.
struct Item {
    int64_t b, d, c;       // sequence and channel of the slab's first; that of the states
    int64_t b0;            // the sequence of its resets, -1 where it has several
    uint32_t slab, place;
    int width;             // channels, or 0: there is nothing left to do
};

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b)
{
    return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// Divisions are dear: one thread works an item out for the block.
__device__ __forceinline__ void set_item(const Args &a, Item &t, uint32_t slab, uint32_t place, bool any)
{
    if (!any) {
        t.width = 0;
        return;
    }
    int64_t left;
    if (a.flat) {
        t.b = 0;
        t.d = (int64_t)slab * kSlab;
        left = a.B * a.D - t.d;
    } else {
        const uint32_t per = (uint32_t)((a.D + kSlab - 1) / kSlab);
        t.b = slab / per;
        t.d = (int64_t)(slab % per) * kSlab;
        left = a.D - t.d;
    }
    t.c = t.b * a.D + t.d;
    t.width = (int)(left < kSlab ? left : kSlab);
    t.b0 = t.b;
    if (a.flat && a.B > 1 && a.reset) {
        t.b0 = divide(t.c, a.D);
        if (t.c + t.width > (t.b0 + 1) * a.D)
            t.b0 = -1;
    }
    t.slab = slab;
    t.place = place;
}

// A chunk in shared memory is [step][64], eight channels' place in a row
// turned by the step's run.
template <int kRun>
__device__ __forceinline__ int place_of(int step, int channel)
{
    return step * kSlab + ((channel >> 3 ^ (step / kRun & 7)) << 3 | (channel & 7));
}

// Calls f(pointer, place) for all of a chunk's pieces of kPer channels that are
// there, dealt to the block's threads; p: the array's first value of the chunk.
template <int kRun, int kPer, class P, class F>
__device__ __forceinline__ void pieces(P *p, int64_t stride, int steps, int width, F f)
{
    constexpr int kAcross = kSlab / kPer, kDown = kThreads / kAcross, kSteps = kRun * kRuns;
    const int channel = threadIdx.x % kAcross * kPer, first = threadIdx.x / kAcross;
    if (channel >= width)
        return;
    p += first * stride + channel;
    if (steps == kSteps) {
#pragma unroll(kSteps / kDown < 8 ? kSteps / kDown : 8)
        for (int k = first; k < kSteps; k += kDown, p += kDown * stride)
            f(p, place_of<kRun>(k, channel));
    } else {
        for (int k = first; k < steps; k += kDown, p += kDown * stride)
            f(p, place_of<kRun>(k, channel));
    }
}

// A chunk of an array to shared memory, as far as there are steps and channels.
template <class T, int kRun>
__device__ __forceinline__ void bring(T *to, const void *from, int64_t st, int64_t sb, const Item &s, int64_t t0,
                                      int steps, int bytes)
{
    const T *p = (const T *)from + t0 * st + s.b * sb + s.d;
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
    if (bytes == 16)
        pieces<kRun, 16 / sizeof(T)>(p, st, steps, s.width, [&](const T *q, int at) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (uint32_t)(at * sizeof(T))), "l"(q)
                         : "memory");
        });
    else if (bytes == 4)
        pieces<kRun, 4 / sizeof(T)>(p, st, steps, s.width, [&](const T *q, int at) {
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + (uint32_t)(at * sizeof(T))), "l"(q)
                         : "memory");
        });
    else
        pieces<kRun, 1>(p, st, steps, s.width, [&](const T *q, int at) { to[at] = *q; });
}

// And back.
template <class T, int kRun>
__device__ __forceinline__ void take_out(const T *from, void *to, int64_t st, int64_t sb, const Item &s, int64_t t0,
                                         int steps, int bytes)
{
    T *p = (T *)to + t0 * st + s.b * sb + s.d;
    if (bytes == 16)
        pieces<kRun, 16 / sizeof(T)>(p, st, steps, s.width, [&](T *q, int at) {
            *reinterpret_cast<uint4 *>(q) = *reinterpret_cast<const uint4 *>(from + at);
        });
    else if (bytes == 4)
        pieces<kRun, 4 / sizeof(T)>(p, st, steps, s.width, [&](T *q, int at) {
            *reinterpret_cast<uint32_t *>(q) = *reinterpret_cast<const uint32_t *>(from + at);
        });
    else
        pieces<kRun, 1>(p, st, steps, s.width, [&](T *q, int at) { *q = from[at]; });
}

// Steps past the sequence's end change nothing: gates of 1, values and
// gradients of 0.
template <class T, int kRun, int kArrays>
__device__ __forceinline__ void pad(T *tile, int steps)
{
    constexpr int kSteps = kRun * kRuns;
    for (int k = steps * kSlab + threadIdx.x; k < kSteps * kSlab; k += kThreads) {
        tile[k] = from_f32<T>(INFINITY);
#pragma unroll
        for (int array = 1; array < kArrays; ++array)
            tile[array * kSteps * kSlab + k] = from_f32<T>(0.0f);
    }
}

template <class T>
__device__ __forceinline__ float2 read2(const T *p)
{
    if constexpr (sizeof(T) == 4)
        return *reinterpret_cast<const float2 *>(p);
    T q[2];
    *reinterpret_cast<uint32_t *>(q) = *reinterpret_cast<const uint32_t *>(p);
    return make_float2(to_f32(q[0]), to_f32(q[1]));
}
template <class T>
__device__ __forceinline__ void write2(T *p, float2 v)
{
    T q[2] = {from_f32<T>(v.x), from_f32<T>(v.y)};
    if constexpr (sizeof(T) == 4)
        *reinterpret_cast<float2 *>(p) = v;
    else
        *reinterpret_cast<uint32_t *>(p) = *reinterpret_cast<const uint32_t *>(q);
}

// v with its sign flipped where bit k (first channel) or 16 + k is set.
__device__ __forceinline__ float2 marked_by(float2 v, uint32_t bits, int k)
{
    v.x = __uint_as_float(__float_as_uint(v.x) ^ (bits << (31 - k) & 0x80000000u));
    v.y = __uint_as_float(__float_as_uint(v.y) ^ (bits << (15 - k) & 0x80000000u));
    return v;
}

// Bits k (first channel) and 16 + k (second) for the steps of this lane's run
// that begin an episode; bits of steps that are not there are 0.
template <int kRun>
__device__ __forceinline__ uint32_t resets_of(const Args &a, const Item &s, int64_t t0, int steps)
{
    if (!a.reset)
        return 0;
    const int lane = threadIdx.x & 31, run = lane >> 2;
    if (s.b0 >= 0) {  // one sequence: the chunk's steps a lane each, four times over
        const uint8_t *p = a.reset + (t0 + lane) * a.rt + s.b0 * a.rb;
        uint32_t mine = 0;
#pragma unroll
        for (int q = 0; q < kRun * kRuns / 32; ++q) {
            const uint32_t m = __ballot_sync(~0u, 32 * q + lane < steps && p[32 * q * a.rt] != 0);
            mine = run * kRun / 32 == q ? m >> (run * kRun % 32) : mine;
        }
        mine &= (1u << kRun) - 1;
        return mine | mine << 16;
    }
    uint32_t m = 0;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const int c = (threadIdx.x >> 5) * 8 + 2 * (lane & 3) + v;
        if (c >= s.width)
            continue;
        const uint8_t *p = a.reset + (t0 + run * kRun) * a.rt + divide(s.c + c, a.D) * a.rb;
        for (int k = 0; k < kRun && run * kRun + k < steps; ++k)
            m |= (p[k * a.rt] != 0 ? 1u : 0u) << (16 * v + k);
    }
    return m;
}

// The state at the start of the chunk at `place` of its chain from the chunks
// before it, and the chunk's own map, `total`, for those after; by each warp
// for its channels.
__device__ void chained(const Args &a, const Item &t, const Map2 &total, int channel, float (&state)[2])
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = lane & 3;
    const uint32_t place = t.place, group = place / kGroup, groups = (a.chunks + kGroup - 1) / kGroup;
    const int before = (int)(place % kGroup);
    const int64_t chain = (int64_t)t.slab * kWarps + warp;
    int *ready = a.ready + chain * a.chunks, *group_ready = a.group_ready + chain * groups;
    float4 *maps = reinterpret_cast<float4 *>(a.maps + chain * a.chunks * 4);
    float2 *group_state = a.group_state + chain * groups * 4;
    if (lane < 4) {
        __stcg(&maps[(int64_t)place * 4 + pair], make_float4(total.A[0], total.A[1], total.H[0], total.H[1]));
        __threadfence();
    }
    __syncwarp();
    if (lane == 0)
        store_flag(ready + place);
    // a flag a lane: the chunks before this one in its group, and the group before
    bool here = true;
    if (lane < before)
        here = wait_flag(ready + (int64_t)group * kGroup + lane, a.limit_ns);
    if (lane == 31 && group > 0)
        here = wait_flag(group_ready + group - 1, a.limit_ns);
    here = __all_sync(~0u, here);
    // four chunks a run of lanes, composed in order, then joined as runs are
    Map2 m = identity();
#pragma unroll
    for (int k = 0; k < kGroup / kRuns; ++k) {
        const int c = (lane >> 2) * (kGroup / kRuns) + k;
        if (c < before) {
            const float4 q = __ldcg(&maps[((int64_t)group * kGroup + c) * 4 + pair]);
            m = then2(m, Map2{{q.x, q.y}, {q.z, q.w}});
        }
    }
    m = whole<false>(joined<false>(m));
    float2 start = make_float2(0.0f, 0.0f);
    if (group > 0) {
        start = __ldcg(&group_state[(int64_t)(group - 1) * 4 + pair]);
    } else if (a.first) {
        start.x = channel < t.width ? a.first[t.c + channel] : 0.0f;
        start.y = channel + 1 < t.width ? a.first[t.c + channel + 1] : 0.0f;
    }
    // (past a wait that ran out all is NaN, so that no wrong state passes for a right one)
    state[0] = here ? apply(m.A[0], m.H[0], start.x) : __int_as_float(0x7fffffff);
    state[1] = here ? apply(m.A[1], m.H[1], start.y) : __int_as_float(0x7fffffff);
    if (before == kGroup - 1) {
        if (lane < 4) {
            __stcg(&group_state[(int64_t)group * 4 + pair], make_float2(apply(total.A[0], total.H[0], state[0]),
                                                                     apply(total.A[1], total.H[1], state[1])));
            __threadfence();
        }
        __syncwarp();
        if (lane == 0)
            store_flag(group_ready + group);
    }
}

// Blocks of an SM: as many as registers and shared memory hold.
__host__ __device__ constexpr int blocks_of(int e, bool back, int run)
{
    return run == kLongRun ? 2 : run == 4 || e == 2 ? 4 : back ? 2 : 3;
}

// kBack: chunks from the last to the first.  What flows to before step t is
// m_t = a_t k_t l_t, l_t = dh_t + m_{t+1}: a run's map of it has the forward
// map's factor.
// kDealt: places are drawn.  The next one is drawn while a chunk's maps are
// made and fetched while its state is waited for, no sooner: a block that sat
// on places would keep those after them waiting.
template <class T, bool kBack, bool kDealt, int kStages, int kRun>
__global__ __launch_bounds__(kThreads, blocks_of(sizeof(T), kBack, kRun)) void scan_kernel(const Args a)
{
    constexpr int kArrays = kBack ? 3 : 2, kChunk = kRun * kRuns, kTile = kChunk * kSlab;
    constexpr int kAhead = kDealt ? 1 : kStages - 1;  // chunks fetched before the first is taken
    extern __shared__ __align__(128) uint8_t raw[];
    __shared__ Item items[4];
    T *tiles = reinterpret_cast<T *>(raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, run = lane >> 2;
    const int channel = warp * 8 + 2 * (lane & 3);
    const int spot = place_of<kRun>(run * kRun, channel);  // of the run's first step; steps are 64 apart

    auto time_of = [&](const Item &t) { return (int64_t)(kBack ? a.chunks - 1 - t.place : t.place) * kChunk; };
    auto steps_at = [&](int64_t t0) { return (int)(a.T - t0 < kChunk ? a.T - t0 : kChunk); };
    auto fill = [&](uint32_t i) {
        const Item &t = items[i & 3];
        if (t.width > 0) {
            const int64_t t0 = time_of(t);
            const int steps = steps_at(t0);
#pragma unroll
            for (int k = 0; k < kArrays; ++k)
                bring<T, kRun>(tiles + (int)(i % kStages * kArrays + k) * kTile, a.in[k], a.it[k], a.ib[k], t, t0, steps,
                               a.in_bytes);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // thread 0: the item after the one it set before
    uint32_t slab_next = blockIdx.x, place_next = 0;
    auto advance = [&](uint32_t i) {
        if (kDealt) {
            const uint32_t drawn = (uint32_t)atomicAdd(a.ticket, 1);
            set_item(a, items[i & 3], drawn % a.slabs, drawn / a.slabs, drawn / a.slabs < a.chunks);
        } else {
            set_item(a, items[i & 3], slab_next, place_next, slab_next < a.slabs);
            if (++place_next == a.chunks) {
                place_next = 0;
                slab_next += gridDim.x;
            }
        }
    };

    if (threadIdx.x == 0)
        for (int i = 0; i <= kAhead - (kDealt ? 1 : 0); ++i)
            advance(i);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        fill(i);
    float carry[2] = {};  // walking: the state that enters the next chunk, in every run's lanes
    for (uint32_t i = 0;; ++i) {
        if (items[i & 3].width == 0)
            break;
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
        __syncthreads();  // this chunk is here, the one before is done with
        if (!kDealt)
            fill(i + kAhead);
        if (threadIdx.x == 0)
            advance(i + kAhead + (kDealt ? 0 : 1));
        const Item item = items[i & 3];
        const int64_t t0 = time_of(item);
        const int steps = steps_at(t0);
        const bool first = channel < item.width, second = channel + 1 < item.width;
        float *kept = a.states ? a.states + t0 / kChunk * (a.B * a.D) + item.c + channel : nullptr;
        T *tile = tiles + (int)(i % kStages) * kArrays * kTile + spot;
        if (steps < kChunk) {
            pad<T, kRun, kArrays>(tiles + (int)(i % kStages) * kArrays * kTile, steps);
            __syncthreads();
        }
        const uint32_t resets = resets_of<kRun>(a, item, t0, steps);
        // (chunks without a reset take no test for one)
        const bool plain = __all_sync(~0u, resets == 0);
        float2 s = make_float2(0.0f, 0.0f);  // forward state before this lane's run
        if (kBack) {
            s.x = first ? kept[0] : 0.0f;
            s.y = second ? kept[1] : 0.0f;
        }
        // the gate, its sign set where an episode begins; 1 - gate (backward) or (1 - gate) v
        float2 ga[kRun], zb[kRun];
        float2 A = make_float2(1.0f, 1.0f), H = make_float2(0.0f, 0.0f), Q = H;
        auto gates = [&](auto simple) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                float2 z;
                gates_of(read2(tile + k * kSlab), ga[k], z);
                const float2 b = mul2(z, read2(tile + kTile + k * kSlab));
                zb[k] = kBack ? z : b;
                A = mul2(A, ga[k]);
                if (simple.value) {
                    H = fma2(ga[k], H, b);
                } else {
                    ga[k] = marked_by(ga[k], resets, k);
                    H = make_float2(apply(ga[k].x, b.x, H.x), apply(ga[k].y, b.y, H.y));
                }
            }
        };
        if (plain)
            gates(std::true_type());
        else
            gates(std::false_type());
        if (resets & 0xffffu)
            A.x = -0.0f;
        if (resets >> 16)
            A.y = -0.0f;
        Map2 m{{A.x, A.y}, {H.x, H.y}}, q = m;  // q, backward: of what flows back
        if (kBack) {
            auto flows = [&](auto simple) {
#pragma unroll
                for (int k = kRun - 1; k >= 0; --k) {
                    Q = mul2(ga[k], add2(read2(tile + 2 * kTile + k * kSlab), Q));
                    if (!simple.value) {
                        Q.x = marked(ga[k].x) ? 0.0f : Q.x;
                        Q.y = marked(ga[k].y) ? 0.0f : Q.y;
                    }
                }
            };
            if (plain)
                flows(std::true_type());
            else
                flows(std::false_type());
            q.H[0] = Q.x;
            q.H[1] = Q.y;
            q = joined<true>(q);
        }
        m = joined<false>(m);
        // what enters the chunk, of the chained direction
        const Map2 total = kBack ? whole<true>(q) : whole<false>(m);
        float in[2];
        if (kDealt) {
            __syncthreads();  // (the next item has been drawn)
            fill(i + 1);
            chained(a, item, total, channel, in);
        } else if (item.place == 0) {
            in[0] = a.first && first ? a.first[item.c + channel] : 0.0f;
            in[1] = a.first && second ? a.first[item.c + channel + 1] : 0.0f;
        } else {
            in[0] = carry[0];
            in[1] = carry[1];
        }
#pragma unroll
        for (int v = 0; v < 2; ++v)
            carry[v] = apply(total.A[v], total.H[v], in[v]);
        if (a.last && item.place == a.chunks - 1 && run == 0) {
            if (first)
                a.last[item.c + channel] = carry[0];
            if (second)
                a.last[item.c + channel + 1] = carry[1];
        }
        if (!kBack) {
            if (kept && run == 0) {
                if (first)
                    kept[0] = in[0];
                if (second)
                    kept[1] = in[1];
            }
            s = make_float2(in[0], in[1]);
        }
        const Map2 pre = before_each<false>(m);
        s.x = apply(pre.A[0], pre.H[0], s.x);
        s.y = apply(pre.A[1], pre.H[1], s.y);
        if (!kBack) {
            auto states = [&](auto simple) {
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    s = simple.value ? fma2(ga[k], s, zb[k])
                                     : make_float2(apply(ga[k].x, zb[k].x, s.x), apply(ga[k].y, zb[k].y, s.y));
                    write2(tile + k * kSlab, s);
                }
            };
            if (plain)
                states(std::true_type());
            else
                states(std::false_type());
        } else {
            const Map2 post = before_each<true>(q);
            // what flows into the run from behind
            float2 f = make_float2(apply(post.A[0], post.H[0], in[0]), apply(post.A[1], post.H[1], in[1]));
            float2 u[kRun];  // v_t - k h_{t-1}
            const float2 minus = make_float2(-1.0f, -1.0f);
            auto gradients = [&](auto simple) {
#pragma unroll
                for (int k = 0; k < kRun; ++k) {
                    const float2 x = read2(tile + kTile + k * kSlab);
                    float2 r = ga[k];
                    if (!simple.value) {
                        s.x = marked(r.x) ? 0.0f : s.x;
                        s.y = marked(r.y) ? 0.0f : s.y;
                        r = make_float2(fabsf(r.x), fabsf(r.y));
                    }
                    u[k] = fma2(s, minus, x);
                    s = fma2(r, s, mul2(zb[k], x));
                }
#pragma unroll
                for (int k = kRun - 1; k >= 0; --k) {
                    const float2 l = add2(read2(tile + 2 * kTile + k * kSlab), f), dv = mul2(zb[k], l);
                    f = mul2(ga[k], l);
                    write2(tile + kTile + k * kSlab, dv);
                    // (f is a l, or -a l where an episode begins)
                    float2 dg = mul2(mul2(f, zb[k]), u[k]);
                    if (simple.value) {
                        dg = mul2(dg, minus);
                    } else {
                        dg.x = marked(ga[k].x) ? dg.x : -dg.x;
                        dg.y = marked(ga[k].y) ? dg.y : -dg.y;
                        f.x = marked(ga[k].x) ? 0.0f : f.x;
                        f.y = marked(ga[k].y) ? 0.0f : f.y;
                    }
                    write2(tile + k * kSlab, dg);
                }
            };
            if (plain)
                gradients(std::true_type());
            else
                gradients(std::false_type());
        }
        __syncthreads();
        const T *done = tiles + (int)(i % kStages) * kArrays * kTile;
#pragma unroll
        for (int k = 0; k < (kBack ? 2 : 1); ++k)
            take_out<T, kRun>(done + k * kTile, a.out[k], a.ot[k], a.ob[k], item, t0, steps, a.out_bytes);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// One step: every value once, kVec at a time.
template <class T, int kVec>
__global__ __launch_bounds__(256) void step_kernel(const Args a)
{
    const int64_t n = a.B * a.D, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * kVec;
    if (c >= n)
        return;
    const int64_t q = c / a.D, d = c % a.D;
    const bool keep = !a.reset || a.reset[q * a.rb] == 0;
    T g[kVec], v[kVec];
    float s[kVec] = {};
    const T *gp = (const T *)a.in[0] + q * a.ib[0] + d, *vp = (const T *)a.in[1] + q * a.ib[1] + d;
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
        float2 r, z;
        gates_of(make_float2(to_f32(g[k]), 0.0f), r, z);
        const float b = z.x * to_f32(v[k]);
        next[k] = keep ? fmaf(r.x, s[k], b) : b;
        o[k] = from_f32<T>(next[k]);
    }
    T *hp = (T *)a.out[0] + q * a.ob[0] + d;
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

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Steps of a run: no more than the sequence has, eight of 32-bit values (two
// blocks' chunks of 16 would not fit shared memory).
int run_of(int64_t T, int e) { return T <= 4 * kRuns ? 4 : T <= 8 * kRuns || e == 4 ? 8 : kLongRun; }
int64_t chunks_of(int64_t T, int e) { return up(T, run_of(T, e) * kRuns); }

// Blocks of channels: numbered through where the sequences lie side by side.
int64_t slabs_of(int64_t B, int64_t D, bool flat) { return flat ? up(B * D, kSlab) : B * up(D, kSlab); }

// Whether chunks are dealt out instead of walked: where walking would leave
// blocks without channels, or the last round of them mostly empty.
bool dealt(int64_t slabs, int64_t chunks, int64_t resident)
{
    if (chunks == 1)
        return false;
    const int64_t rounds = up(slabs, resident);
    return rounds * resident * 8 > slabs * 9;
}

int64_t flag_bytes(int64_t slabs, int64_t chunks) { return up((1 + slabs * kWarps * (chunks + up(chunks, kGroup))) * 4, 256) * 256; }

int64_t plan_bytes(int64_t slabs, int64_t chunks)
{
    return flag_bytes(slabs, chunks) + slabs * kWarps * 4 * (chunks * (int64_t)sizeof(Map2) + up(chunks, kGroup) * 8);
}

int64_t work_bytes(int64_t T, int64_t B, int64_t D, int e)
{
    const int64_t chunks = chunks_of(T, e);
    int64_t most = 0;
    for (int flat = 0; flat < 2; ++flat)
        for (int back = 0; back < 2; ++back) {
            const int64_t slabs = slabs_of(B, D, flat);
            const int64_t need = T > 1 && dealt(slabs, chunks, kSms * blocks_of(e, back, run_of(T, e))) ? plan_bytes(slabs, chunks) : 0;
            most = need > most ? need : most;
        }
    return most;
}

// How an array's values can be copied, given those before it: 16 or 4 bytes at
// once, or one by one (0).  A copy reads no further than the array's own row.
int copy_bytes(int so_far, const void *p, int64_t t, int64_t b, int64_t n, int e)
{
    auto fits = [&](int bytes) {
        return so_far >= bytes && (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0 && t * e % bytes == 0 &&
               b * e % bytes == 0 && n * e % bytes == 0;
    };
    return fits(16) ? 16 : fits(4) ? 4 : 0;
}

template <class T, bool kBack, int kRun>
cudaError_t go(Args &a, void *work, cudaStream_t st)
{
    constexpr int kArrays = kBack ? 3 : 2, kOut = kBack ? 2 : 1, kStages = kBack || sizeof(T) == 4 ? 2 : 3;
    constexpr int kBytes = kStages * kArrays * kRun * kRuns * kSlab * (int)sizeof(T);
    const int64_t chunks = chunks_of(a.T, sizeof(T));
    a.flat = true;
    for (int k = 0; k < kArrays; ++k)
        a.flat = a.flat && (a.B == 1 || a.ib[k] == a.D);
    for (int k = 0; k < kOut; ++k)
        a.flat = a.flat && (a.B == 1 || a.ob[k] == a.D);
    const int64_t slabs = slabs_of(a.B, a.D, a.flat);
    if (slabs * chunks > (int64_t(1) << 31))  // (beyond any memory)
        return cudaErrorInvalidValue;
    a.slabs = (uint32_t)slabs;
    a.chunks = (uint32_t)chunks;
    const int64_t n = a.flat ? a.B * a.D : a.D;
    a.in_bytes = a.out_bytes = 16;
    for (int k = 0; k < kArrays; ++k)
        a.in_bytes = copy_bytes(a.in_bytes, a.in[k], a.it[k], a.flat ? 0 : a.ib[k], n, sizeof(T));
    for (int k = 0; k < kOut; ++k)
        a.out_bytes = copy_bytes(a.out_bytes, a.out[k], a.ot[k], a.flat ? 0 : a.ob[k], n, sizeof(T));
    constexpr int64_t resident = kSms * blocks_of(sizeof(T), kBack, kRun);
    int64_t grid = slabs < resident ? slabs : resident;
    if (dealt(slabs, chunks, resident)) {
        const int64_t flags = flag_bytes(slabs, chunks), items = slabs * chunks;
        grid = items < resident ? items : resident;
        a.ticket = (int *)work;
        a.ready = a.ticket + 1;
        a.group_ready = a.ready + slabs * kWarps * chunks;
        a.maps = (Map2 *)((char *)work + flags);
        a.group_state = (float2 *)(a.maps + slabs * kWarps * chunks * 4);
        a.limit_ns = 4000000000ll;
        if (const char *ms = getenv("AV_SCAN_WAIT_MS"))  // for tests of the limit
            a.limit_ns = atoll(ms) * 1000000;
        const cudaError_t e = cudaMemsetAsync(work, 0, flags, st);
        if (e != cudaSuccess)
            return e;
    }
    auto run = [&](auto kernel) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
        if (e != cudaSuccess)
            return e;
        kernel<<<(unsigned)grid, kThreads, kBytes, st>>>(a);
        return cudaGetLastError();
    };
    if constexpr (kRun == (sizeof(T) == 4 ? 8 : kLongRun)) {
        if (a.ticket)
            return run(scan_kernel<T, kBack, true, kStages, kRun>);
    }
    return run(scan_kernel<T, kBack, false, kStages, kRun>);
}

template <bool kBack>
cudaError_t launch(Args &a, int dtype, void *work, cudaStream_t st)
{
    return with_type(dtype, [&](auto v) {
        using T = decltype(v);
        const int run = run_of(a.T, sizeof(T));
        if constexpr (sizeof(T) == 2) {
            if (run == kLongRun)
                return go<T, kBack, kLongRun>(a, work, st);
        }
        return run == 4 ? go<T, kBack, 4>(a, work, st) : go<T, kBack, 8>(a, work, st);
    });
}

}  // namespace

void scan_sizes(int64_t T, int64_t B, int64_t D, int dtype, int64_t *states, int64_t *work)
{
    const int e = dtype == AV_F32 ? 4 : 2;
    *states = chunks_of(T, e) * B * D;
    *work = work_bytes(T, B, D, e);
}

cudaError_t launch_scan(int64_t T, int64_t B, int64_t D, int dtype, Seq gate, Seq value, Seq reset, const float *h0,
                        SeqOut h, float *h_last, float *states, void *work, cudaStream_t st)
{
    Args a{};
    a.T = T, a.B = B, a.D = D;
    a.in[0] = gate.p, a.it[0] = gate.t, a.ib[0] = gate.b;
    a.in[1] = value.p, a.it[1] = value.t, a.ib[1] = value.b;
    a.reset = (const uint8_t *)reset.p, a.rt = reset.t, a.rb = reset.b;
    a.out[0] = h.p, a.ot[0] = h.t, a.ob[0] = h.b;
    a.first = h0, a.last = h_last, a.states = states;
    if (T > 1)
        return launch<false>(a, dtype, work, st);
    const int64_t n = B * D;
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

cudaError_t launch_scan_grad(int64_t T, int64_t B, int64_t D, int dtype, Seq dh, Seq gate, Seq value, Seq reset,
                             const float *states, const float *dlast, SeqOut dgate, SeqOut dvalue, float *dh0,
                             void *work, cudaStream_t st)
{
    Args a{};
    a.T = T, a.B = B, a.D = D;
    a.in[0] = gate.p, a.it[0] = gate.t, a.ib[0] = gate.b;
    a.in[1] = value.p, a.it[1] = value.t, a.ib[1] = value.b;
    a.in[2] = dh.p, a.it[2] = dh.t, a.ib[2] = dh.b;
    a.reset = (const uint8_t *)reset.p, a.rt = reset.t, a.rb = reset.b;
    a.out[0] = dgate.p, a.ot[0] = dgate.t, a.ob[0] = dgate.b;
    a.out[1] = dvalue.p, a.ot[1] = dvalue.t, a.ob[1] = dvalue.b;
    a.first = dlast, a.last = dh0, a.states = const_cast<float *>(states);
    return launch<true>(a, dtype, work, st);
}

}  // namespace av
