// k_scan.cu -- the gated linear recurrence and its gradient.
//   forward   a = sigmoid(g), h_t = a k_t h_{t-1} + (1 - a) v_t
//   backward  l_t = dh_t + a_{t+1} k_{t+1} l_{t+1}; dv = (1 - a) l; dg = l (k h_{t-1} - v) a (1 - a)
//
// Steps are affine maps h -> A h + H, and maps compose: a run of steps is one
// map whatever its length.  A block takes 64 channels and chunks of 128 steps
// (64 of 32-bit values, 32 or 64 of shorter sequences).  A warp takes eight of
// the channels: its lanes are four pairs of them by eight runs of 16 steps, so
// that runs are joined by shuffles and no warp waits for another.  Chunks come
// and go by TMA through shared memory, the next one under way during this one,
// results leaving from the places of the inputs they came from.  The tensor
// maps lay step k of all eight runs side by side, so that the 128-byte swizzle
// sends lanes of different runs to different banks.  (A chunk that reaches past
// the sequence goes by cp.async, to the same places.)  Arrays that TMA does not
// take, of odd widths or strides, come row by row by bulk copies of the 16-byte
// pieces that hold a row's values.  Both directions read and write their arrays
// once: 3 and 5 values a step and channel.  The backward pass makes the states
// again from the one kept at each chunk's start (4 bytes a chunk and channel),
// so it neither reads h nor suffers its rounding.  Bound by memory, and for
// 16-bit values by issue.
//
// A block walks its channels' chunks in order.  Where the channels would not
// fill the GPU, a sequence is cut into segments: a first pass makes every
// segment's map, a second walks the segments from the states that the maps
// before them give, in one order.  The inputs are read twice then, but no block
// waits for another.  Up to eight steps (16 of 32 bits) of many channels take a
// thread for two channels.
//
// A step that begins an episode forgets the state even where it is NaN: in a
// map this is a factor with its sign bit set, which survives composition.
#include <type_traits>

#include "async.cuh"
#include "policy.h"
#include "tensor_map.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kRuns = 8;         // runs of a chunk, a quarter of a warp's lanes each
constexpr int kLongRun = 16;     // steps of a run at most
constexpr int kSlab = 64;        // channels of a block, eight a warp, two a lane
constexpr int kSms = 152;
constexpr int kMaps = 32;        // maps of a block: a pair of channels each
// From where on brief sequences take a thread for two channels: of 16,384 four
// steps take 4.6 us so and 6.5 walked, eight 6.7 and 6.5 (backward 6.7 and 8.5),
// of 131,072 channels eight 6.7 and 19.8.
constexpr int64_t kBriefChannels = 4096;

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
    uint32_t segments, per;     // segments of a sequence, chunks of a segment
    Map2 *maps;                 // [slab][segment][kMaps], where there are several segments
    bool flat;                  // sequences lie side by side: channels are numbered through
    int words[2];               // of the outputs: whether 32-bit words of them can be stored
};
// The arrays for TMA: inputs, outputs.
struct TensorMaps {
    CUtensorMap in[3], out[2];
};

// What a block does next: chunk `place` chunks after its chain's first
// (backward: from the end) of a slab of channels.
struct Item {
    int64_t b, d, c;       // sequence and channel of the slab's first; that of the states
    int64_t b0;            // the sequence of its resets, -1 where it has several
    uint32_t slab, segment, place;
    bool enters;           // the segment's first chunk
    int width;             // channels, or 0: there is nothing left to do
};

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b)
{
    return (a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// Divisions are dear: one thread works an item out for the block.
__device__ __forceinline__ void set_item(const Args &a, Item &t, uint32_t unit, uint32_t place)
{
    t.slab = unit / a.segments;
    if (t.slab >= a.slabs) {
        t.width = 0;
        return;
    }
    t.segment = unit - t.slab * a.segments;
    t.place = place;
    t.enters = place == t.segment * a.per;
    int64_t left;
    if (a.flat) {
        t.b = 0;
        t.d = (int64_t)t.slab * kSlab;
        left = a.B * a.D - t.d;
    } else {
        const uint32_t across = (uint32_t)((a.D + kSlab - 1) / kSlab);
        t.b = t.slab / across;
        t.d = (int64_t)(t.slab % across) * kSlab;
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
}

// The order of a block's items: units (a segment of a slab) gridDim.x apart,
// the chunks of each in order.
struct Order {
    uint32_t unit, place, end;
    __device__ __forceinline__ void open(const Args &a)
    {
        const uint32_t segment = unit % a.segments;
        place = segment * a.per;
        end = place + a.per < a.chunks ? place + a.per : a.chunks;
    }
    __device__ __forceinline__ void next(const Args &a, Item &t)
    {
        set_item(a, t, unit, place);
        if (++place >= end) {
            unit += gridDim.x;
            open(a);
        }
    }
};

// A chunk of an array in shared memory: rows of 128 bytes, step k of run r in
// row 8 k + r, its 16-byte pieces turned by r (the 128-byte swizzle).  32-bit
// values are two such blocks of 32 channels.
template <class T, int kRun>
__device__ __forceinline__ int place_of(int step, int channel)
{
    const int r = step / kRun, row = step % kRun * kRuns + r;
    if constexpr (sizeof(T) == 4)
        return (channel >> 5) * (kRun * kRuns * 32) + row * 32 + (((channel & 31) >> 2 ^ r) << 2 | (channel & 3));
    return row * 64 + ((channel >> 3 ^ r) << 3 | (channel & 7));
}
// Values between a run's steps.
template <class T>
__device__ constexpr int step_of() { return kRuns * 128 / (int)sizeof(T); }

// f(pointer, place) for the 16-byte pieces of a chunk that are there, dealt to
// the block's threads; p: the array's first value of the chunk.
template <class T, int kRun, class P, class F>
__device__ __forceinline__ void pieces(P *p, int64_t stride, int steps, int width, F f)
{
    constexpr int kPer = 16 / sizeof(T), kAcross = kSlab / kPer, kDown = kThreads / kAcross;
    const int channel = threadIdx.x % kAcross * kPer, first = threadIdx.x / kAcross;
    if (channel >= width)
        return;
    p += first * stride + channel;
#pragma unroll 2
    for (int k = first; k < steps; k += kDown, p += kDown * stride)
        f(p, place_of<T, kRun>(k, channel));
}

// A chunk of an array to shared memory, as far as there are steps and channels.
template <class T, int kRun>
__device__ __noinline__ void bring(T *to, const void *from, int64_t st, int64_t sb, const Item &s, int64_t t0, int steps)
{
    const uint32_t dst = smem_addr(to);
    pieces<T, kRun>((const T *)from + t0 * st + s.b * sb + s.d, st, steps, s.width, [&](const T *q, int at) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (uint32_t)(at * sizeof(T))), "l"(q)
                     : "memory");
    });
}

// And back.
template <class T, int kRun>
__device__ __noinline__ void take_out(const T *from, void *to, int64_t st, int64_t sb, const Item &s, int64_t t0,
                                      int steps)
{
    pieces<T, kRun>((T *)to + t0 * st + s.b * sb + s.d, st, steps, s.width, [&](T *q, int at) {
        *reinterpret_cast<uint4 *>(q) = *reinterpret_cast<const uint4 *>(from + at);
    });
}

// Rows by bulk copies: bytes from one row to the next, an odd number of 16-byte
// pieces, so that runs' rows, side by side, are in different banks.
template <class T>
__host__ __device__ constexpr int pitch_of() { return kSlab * (int)sizeof(T) + 16; }
template <class T, int kRun>
__host__ __device__ constexpr int rows_bytes() { return kRun * kRuns * pitch_of<T>(); }
// The row of a step.
template <int kRun>
__device__ __forceinline__ int row_of(int step) { return step % kRun * kRuns + step / kRun; }

// This thread's rows of a chunk's arrays to shared memory; it arrives at the
// barrier with their bytes.
template <class T, int kRun, int kArrays>
__device__ __forceinline__ void bring_rows(uint32_t to, const Args &a, const int (&array)[kArrays], const Item &s,
                                           int64_t t0, int steps, uint32_t bar)
{
    constexpr int kChunk = kRun * kRuns, kTurns = (kArrays * kChunk + kThreads - 1) / kThreads;
    const char *from[kTurns];
    uint32_t bytes[kTurns], all = 0;
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
        const int row = threadIdx.x + j * kThreads, k = row / kChunk, t = row % kChunk;
        bytes[j] = 0;
        if (k < kArrays && t < steps) {
            const void *p = a.in[array[0]];
            int64_t st = a.it[array[0]], sb = a.ib[array[0]];
#pragma unroll
            for (int q = 1; q < kArrays; ++q)
                if (k == q) {
                    p = a.in[array[q]];
                    st = a.it[array[q]];
                    sb = a.ib[array[q]];
                }
            const T *first = (const T *)p + (t0 + t) * st + s.b * sb + s.d;
            const uint32_t lead = (uint32_t)reinterpret_cast<uintptr_t>(first) & 15;
            from[j] = reinterpret_cast<const char *>(first) - lead;
            bytes[j] = (lead + s.width * (uint32_t)sizeof(T) + 15) & ~15u;
            all += bytes[j];
        }
    }
    bar_expect(bar, all);
#pragma unroll
    for (int j = 0; j < kTurns; ++j) {
        const int row = threadIdx.x + j * kThreads;
        if (bytes[j])
            bulk_load(to + (row / kChunk) * rows_bytes<T, kRun>() + row_of<kRun>(row % kChunk) * pitch_of<T>(), from[j],
                      bytes[j], bar);
    }
}

// The bytes before a row's first value, of step t from the chunk's start.
template <class T>
__device__ __forceinline__ uint32_t lead_of(const void *p, int64_t st, int64_t sb, const Item &s, int64_t t)
{
    return (uint32_t)reinterpret_cast<uintptr_t>((const T *)p + t * st + s.b * sb + s.d) & 15;
}

// Results, in the places of array k's rows (whose leads they have), out.
template <class T, int kRun>
__device__ __noinline__ void rows_out(const char *from, const Args &a, int k, const Item &s, int64_t t0, int steps)
{
    const char *rows = from + k * rows_bytes<T, kRun>();
    T *p = (T *)a.out[k] + t0 * a.ot[k] + s.b * a.ob[k] + s.d;
    const uint32_t lead0 = lead_of<T>(a.in[k], a.it[k], a.ib[k], s, t0), step = (uint32_t)(a.it[k] * sizeof(T)) & 15;
    if (sizeof(T) == 2 && a.words[k]) {  // a word of two values a lane, a row a warp
        const int c = (threadIdx.x & 31) * 2;
#pragma unroll 4
        for (int t = threadIdx.x >> 5; t < steps; t += kWarps) {
            const T *q = reinterpret_cast<const T *>(rows + row_of<kRun>(t) * pitch_of<T>() + ((lead0 + t * step) & 15)) + c;
            const T v[2] = {q[0], q[1]};
            if (c + 1 < s.width)
                *reinterpret_cast<uint32_t *>(p + t * a.ot[k] + c) = *reinterpret_cast<const uint32_t *>(v);
            else if (c < s.width)
                p[t * a.ot[k] + c] = v[0];
        }
        return;
    }
    const int c = threadIdx.x % kSlab;
#pragma unroll 4
    for (int t = threadIdx.x / kSlab; t < steps; t += kThreads / kSlab)
        if (c < s.width)
            p[t * a.ot[k] + c] =
                reinterpret_cast<const T *>(rows + row_of<kRun>(t) * pitch_of<T>() + ((lead0 + t * step) & 15))[c];
}

// Steps past the sequence's end change nothing: gates of 1, values and
// gradients of 0.
template <class T, int kRun>
__device__ __noinline__ void pad(T *tile, int steps, int arrays)
{
    constexpr int kSteps = kRun * kRuns;
    for (int k = steps * kSlab + threadIdx.x; k < kSteps * kSlab; k += kThreads) {
        const int at = place_of<T, kRun>(k / kSlab, k % kSlab);
        tile[at] = from_f32<T>(INFINITY);
        for (int array = 1; array < arrays; ++array)
            tile[array * kSteps * kSlab + at] = from_f32<T>(0.0f);
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

// The same for rows, whatever their leads.
template <class T, int kRun>
__device__ __noinline__ void pad_rows(char *tile, int steps, int arrays)
{
    constexpr int kPer = pitch_of<T>() / (int)sizeof(T);
    for (int k = steps * kPer + threadIdx.x; k < kRun * kRuns * kPer; k += kThreads) {
        const int at = row_of<kRun>(k / kPer) * kPer + k % kPer;
        for (int array = 0; array < arrays; ++array)
            reinterpret_cast<T *>(tile + array * rows_bytes<T, kRun>())[at] = from_f32<T>(array == 0 ? INFINITY : 0.0f);
    }
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
        uint8_t begins[kRun * kRuns / 32];
#pragma unroll
        for (int q = 0; q < kRun * kRuns / 32; ++q)
            begins[q] = 32 * q + lane < steps ? p[32 * q * a.rt] : 0;
        uint32_t mine = 0;
#pragma unroll
        for (int q = 0; q < kRun * kRuns / 32; ++q) {
            const uint32_t m = __ballot_sync(~0u, begins[q] != 0);
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

// A run's values in shared memory: array 0 holds gates (then h or their
// gradients), 1 values (their gradients), 2 dh.
template <class T, int kRun>
struct Tile {
    T *p;
    __device__ __forceinline__ float2 get(int array, int k) const
    {
        return read2(p + array * (kRun * kRuns * kSlab) + k * step_of<T>());
    }
    __device__ __forceinline__ void put(int array, int k, float2 v) const
    {
        write2(p + array * (kRun * kRuns * kSlab) + k * step_of<T>(), v);
    }
};

// The same where rows came by bulk copies: each has its lead.  kPairs: of whole
// 32-bit words, so that two 16-bit values are one.
template <class T, int kRun, int kArrays, bool kPairs>
struct Rows {
    char *p;  // the run's first row and the lane's channel, without a lead
    uint32_t lead[kArrays], step[kArrays];
    __device__ __forceinline__ T *at(int array, int k) const
    {
        return reinterpret_cast<T *>(p + array * rows_bytes<T, kRun>() + k * kRuns * pitch_of<T>() +
                                     ((lead[array] + k * step[array]) & 15));
    }
    __device__ __forceinline__ float2 get(int array, int k) const
    {
        const T *q = at(array, k);
        if constexpr (kPairs)
            return read2(q);
        return make_float2(to_f32(q[0]), to_f32(q[1]));
    }
    __device__ __forceinline__ void put(int array, int k, float2 v) const
    {
        T *q = at(array, k);
        if constexpr (kPairs) {
            write2(q, v);
        } else {
            q[0] = from_f32<T>(v.x);
            q[1] = from_f32<T>(v.y);
        }
    }
};

// A run's steps in a lane's registers.
template <bool kBack, int kRun>
struct Run {
    uint32_t resets;  // steps that begin an episode, as resets_of gives them
    bool plain;       // none in the warp: steps take no test for one
    // the gate, its sign set where an episode begins; 1 - gate (backward) or (1 - gate) v
    float2 ga[kRun], zb[kRun];

    // Fills ga and zb; the run's map of the state.
    template <class Tile>
    __device__ __forceinline__ Map2 gates(const Tile &tile)
    {
        float2 A = make_float2(1.0f, 1.0f), H = make_float2(0.0f, 0.0f);
        auto go = [&](auto simple) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                float2 z;
                gates_of(tile.get(0, k), ga[k], z);
                const float2 b = mul2(z, tile.get(1, k));
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
            go(std::true_type());
        else
            go(std::false_type());
        return {{resets & 0xffffu ? -0.0f : A.x, resets >> 16 ? -0.0f : A.y}, {H.x, H.y}};
    }

    // Backward, after gates: the run's map of what flows back, its factors those of `map`.
    template <class Tile>
    __device__ __forceinline__ Map2 flows(const Tile &tile, const Map2 &map) const
    {
        float2 Q = make_float2(0.0f, 0.0f);
        auto go = [&](auto simple) {
#pragma unroll
            for (int k = kRun - 1; k >= 0; --k) {
                Q = mul2(ga[k], add2(tile.get(2, k), Q));
                if (!simple.value) {
                    Q.x = marked(ga[k].x) ? 0.0f : Q.x;
                    Q.y = marked(ga[k].y) ? 0.0f : Q.y;
                }
            }
        };
        if (plain)
            go(std::true_type());
        else
            go(std::false_type());
        return {{map.A[0], map.A[1]}, {Q.x, Q.y}};
    }

    // Backward, alone: the map of what flows back, without values.
    template <class Tile>
    __device__ __forceinline__ Map2 flow_map(const Tile &tile) const
    {
        float2 A = make_float2(1.0f, 1.0f), Q = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = kRun - 1; k >= 0; --k) {
            float2 g, z;
            gates_of(tile.get(0, k), g, z);
            A = mul2(A, g);
            Q = mul2(g, add2(tile.get(1, k), Q));
            Q.x = resets >> k & 1 ? 0.0f : Q.x;
            Q.y = resets >> (16 + k) & 1 ? 0.0f : Q.y;
        }
        return {{resets & 0xffffu ? -0.0f : A.x, resets >> 16 ? -0.0f : A.y}, {Q.x, Q.y}};
    }

    // Forward: the states, to the gates' places; s is the one before the run.
    template <class Tile>
    __device__ __forceinline__ void states(const Tile &tile, float2 s) const
    {
        auto go = [&](auto simple) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                s = simple.value ? fma2(ga[k], s, zb[k])
                                 : make_float2(apply(ga[k].x, zb[k].x, s.x), apply(ga[k].y, zb[k].y, s.y));
                tile.put(0, k, s);
            }
        };
        if (plain)
            go(std::true_type());
        else
            go(std::false_type());
    }

    // Backward: the gradients, to the gates' and the values' places; f flows
    // into the run from behind.
    template <class Tile>
    __device__ __forceinline__ void gradients(const Tile &tile, float2 s, float2 f) const
    {
        float2 u[kRun];  // v_t - k h_{t-1}
        const float2 minus = make_float2(-1.0f, -1.0f);
        auto go = [&](auto simple) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                const float2 x = tile.get(1, k);
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
                const float2 l = add2(tile.get(2, k), f), dv = mul2(zb[k], l);
                f = mul2(ga[k], l);
                tile.put(1, k, dv);
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
                tile.put(0, k, dg);
            }
        };
        if (plain)
            go(std::true_type());
        else
            go(std::false_type());
    }
};

// A block's view of a chunk.
struct Chunk {
    int64_t t0;
    uint32_t index;
    int steps;
    bool first, second;  // whether the lane's two channels are there
    __device__ __forceinline__ float *kept(const Args &a, const Item &t, int channel) const
    {
        return a.states + index * (a.B * a.D) + t.c + channel;
    }
};
template <bool kBack, int kSteps>
__device__ __forceinline__ Chunk chunk_of(const Args &a, const Item &t, int channel)
{
    Chunk c;
    c.index = kBack ? a.chunks - 1 - t.place : t.place;
    c.t0 = (int64_t)c.index * kSteps;
    c.steps = (int)(a.T - c.t0 < kSteps ? a.T - c.t0 : kSteps);
    c.first = channel < t.width;
    c.second = channel + 1 < t.width;
    return c;
}

// The state that enters a segment: the first one through the maps of the
// segments before it, eight lanes' shares of them in order.
__device__ __noinline__ float2 entering(const Args &a, const Item &t, int channel)
{
    const int lane = threadIdx.x & 31, run = lane >> 2, pair = (threadIdx.x >> 5) * 4 + (lane & 3);
    float2 s = make_float2(0.0f, 0.0f);
    if (a.first) {
        s.x = channel < t.width ? a.first[t.c + channel] : 0.0f;
        s.y = channel + 1 < t.width ? a.first[t.c + channel + 1] : 0.0f;
    }
    if (t.segment == 0)
        return s;
    const float4 *maps = reinterpret_cast<const float4 *>(a.maps + (int64_t)t.slab * a.segments * kMaps + pair);
    const uint32_t share = (t.segment + kRuns - 1) / kRuns;
    Map2 m = identity();
#pragma unroll 4
    for (uint32_t k = run * share; k < (run + 1) * share && k < t.segment; ++k) {
        const float4 q = maps[(int64_t)k * kMaps];
        m = then2(m, Map2{{q.x, q.y}, {q.z, q.w}});
    }
    m = whole<false>(joined<false>(m));
    return make_float2(apply(m.A[0], m.H[0], s.x), apply(m.A[1], m.H[1], s.y));
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, int c, int run, int b, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
                 "l"(map), "r"(c), "r"(run), "r"(0), "r"(b), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, uint32_t src, int c, int run, int b)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(map),
                 "r"(src), "r"(c), "r"(run), "r"(0), "r"(b)
                 : "memory");
}

// Blocks of an SM: as many as registers and shared memory hold.
__host__ __device__ constexpr int blocks_of(int e, bool back, int run)
{
    return run == kLongRun ? 2 : run == 4 ? 4 : back ? 2 : 3;
}
// Chunks in shared memory: the one that is taken and the next; forward by TMA
// also one whose results are leaving.
__host__ __device__ constexpr int stages_of(int e, bool back, bool maps_only, bool tma)
{
    return e == 4 || back || maps_only || !tma ? 2 : 3;
}
// Bytes of an array's chunk.
template <class T, int kRun>
__host__ __device__ constexpr int chunk_bytes(bool tma)
{
    return tma ? kRun * kRuns * kSlab * (int)sizeof(T) : rows_bytes<T, kRun>();
}

// How chunks come: by TMA, or row by row, of pairs of 16-bit values or singly.
enum Way { kByTma, kByPairs, kBySingles };

// kBack: chunks from the last to the first.  What flows to before step t is
// m_t = a_t k_t l_t, l_t = dh_t + m_{t+1}: a run's map of it has the forward
// map's factor.
// kMapsOnly: no outputs but the segments' maps (backward these take gates and
// dh alone).
// 128 steps of 1,024 x 256 16-bit values take 60 us forward and 96 back, 3.4 and
// 3.5 TB/s: two blocks of 128 registers a thread are resident, warps wait for
// chunks half of the time and issue 1.9 and 1.7 of 4 instructions a cycle.
// 65,537 steps of 1,021 32-bit channels, in segments, 304 and 504 us.
template <class T, bool kBack, bool kMapsOnly, int kWay, int kRun>
__global__ __launch_bounds__(kThreads, blocks_of(sizeof(T), kBack, kRun)) void walk_kernel(
    const __grid_constant__ TensorMaps tma, const Args a)
{
    constexpr int kArrays = kBack && !kMapsOnly ? 3 : 2, kOut = kMapsOnly ? 0 : kBack ? 2 : 1;
    constexpr bool kTma = kWay == kByTma;
    constexpr int kChunk = kRun * kRuns, kStages = stages_of(sizeof(T), kBack, kMapsOnly, kTma);
    constexpr int kBytes = chunk_bytes<T, kRun>(kTma);            // of an array's chunk
    constexpr int kBoxes = sizeof(T) / 2, kBox = kBytes / kBoxes;  // of it by TMA; bytes of one
    extern __shared__ uint8_t raw[];
    __shared__ Item items[4];
    __shared__ uint64_t bars[kStages];
    __shared__ int dead;
    char *tiles = reinterpret_cast<char *>(raw + ((1024 - (smem_addr(raw) & 1023)) & 1023));
    const int channel = (threadIdx.x >> 5) * 8 + 2 * (threadIdx.x & 3), run_at = (threadIdx.x & 31) / 4 * kRun;
    auto stage = [&](int s, int k = 0) { return tiles + (s * kArrays + k) * kBytes; };
    // which of the call's arrays are the tile's
    const int arrays[3] = {0, kBack && kMapsOnly ? 2 : 1, 2};
    auto time_of = [&](const Item &t) { return (int64_t)(kBack ? a.chunks - 1 - t.place : t.place) * kChunk; };
    auto steps_at = [&](int64_t t0) { return (int)(a.T - t0 < kChunk ? a.T - t0 : kChunk); };
    auto by_tma = [&](const Item &t) { return kTma && a.T - time_of(t) >= kChunk; };
    // all threads: an item's chunk to stage s
    auto fill = [&](const Item &t, int s) {
        if (t.width > 0) {
            const int64_t t0 = time_of(t);
            const uint32_t bar = smem_addr(bars + s);
            if constexpr (!kTma) {
                int which[kArrays];
#pragma unroll
                for (int k = 0; k < kArrays; ++k)
                    which[k] = arrays[k];
                bring_rows<T, kRun, kArrays>(smem_addr(stage(s)), a, which, t, t0, steps_at(t0), bar);
            } else if (by_tma(t)) {
                if (threadIdx.x == 0) {
                    // (what left from this stage has been read)
                    if constexpr (kOut > 0)
                        asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kStages - 2) : "memory");
                    bar_expect(bar, kArrays * kBytes);
#pragma unroll
                    for (int k = 0; k < kArrays; ++k)
#pragma unroll
                        for (int q = 0; q < kBoxes; ++q)
                            tma_load(smem_addr(stage(s, k)) + q * kBox, &tma.in[arrays[k]],
                                     (int)t.d + q * (kSlab / kBoxes), (int)(t0 / kRun), (int)t.b, bar);
                }
            } else {
                if (kOut > 0) {
                    if (threadIdx.x == 0)
                        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncthreads();
                }
#pragma unroll
                for (int k = 0; k < kArrays; ++k) {
                    const int q = arrays[k];
                    bring<T, kRun>(reinterpret_cast<T *>(stage(s, k)), a.in[q], a.it[q], a.ib[q], t, t0, steps_at(t0));
                }
            }
        }
        if (kTma)
            asm volatile("cp.async.commit_group;" ::: "memory");
    };
    Order order{blockIdx.x, 0, 0};  // thread 0's
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < kStages; ++s)
            bar_init(smem_addr(bars + s), kTma ? 1 : kThreads);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        order.open(a);
        order.next(a, items[0]);
        order.next(a, items[1]);
    }
    __syncthreads();
    if constexpr (kMapsOnly)
        next_may_start();
    else
        after_previous();
    fill(items[0], 0);
    bool ok = true;
    uint32_t phases = 0;
    Map2 all = identity();     // the segment's map so far
    float carry[2] = {};       // the state that enters the next chunk, in every run's lanes
    int s = 0;
    for (uint32_t i = 0; items[i & 3].width > 0; ++i) {
        if (!kTma || by_tma(items[i & 3])) {
            ok = ok && bar_wait(smem_addr(bars + s), phases >> s & 1, &dead);
            phases ^= 1u << s;
        }
        if (kTma)
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (before copies to where this thread read or wrote)
        ok = __syncthreads_and(ok);  // this chunk is here, the one before is done with
        const int s_next = s + 1 == kStages ? 0 : s + 1;
        if (ok) {
            fill(items[(i + 1) & 3], s_next);
        } else if (kTma && kOut > 0) {  // (what left from this stage has been read)
            if (threadIdx.x == 0)
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncthreads();
        }
        if (threadIdx.x == 0)
            order.next(a, items[(i + 2) & 3]);
        const Item item = items[i & 3];
        const Chunk c = chunk_of<kBack, kChunk>(a, item, channel);
        if (c.steps < kChunk) {
            if (kTma)
                pad<T, kRun>(reinterpret_cast<T *>(stage(s)), c.steps, kArrays);
            else
                pad_rows<T, kRun>(stage(s), c.steps, kArrays);
            __syncthreads();
        }
        const auto tile = [&] {
            if constexpr (kTma) {
                return Tile<T, kRun>{reinterpret_cast<T *>(stage(s)) + place_of<T, kRun>(run_at, channel)};
            } else {
                Rows<T, kRun, kArrays, kWay == kByPairs> rows;
                rows.p = stage(s) + (run_at / kRun) * pitch_of<T>() + channel * sizeof(T);
#pragma unroll
                for (int k = 0; k < kArrays; ++k) {
                    const int q = arrays[k];
                    rows.lead[k] = lead_of<T>(a.in[q], a.it[q], a.ib[q], item, c.t0 + run_at);
                    rows.step[k] = (uint32_t)(a.it[q] * sizeof(T)) & 15;
                }
                return rows;
            }
        }();
        Run<kBack, kRun> run;
        // (past a wait that ran out nothing is known of the steps, and no begin of an episode ends the NaN)
        run.resets = ok ? resets_of<kRun>(a, item, c.t0, c.steps) : 0;
        run.plain = __all_sync(~0u, run.resets == 0);
        if constexpr (kMapsOnly) {
            const Map2 m = kBack ? whole<true>(joined<true>(run.flow_map(tile))) : whole<false>(joined<false>(run.gates(tile)));
            all = item.enters ? m : then2(all, m);
            const uint32_t end = (item.segment + 1) * a.per;
            if (item.place + 1 == (end < a.chunks ? end : a.chunks) && (threadIdx.x & 31) < 4) {
                if (!ok)
                    all = Map2{{-0.0f, -0.0f}, {__int_as_float(0x7fffffff), __int_as_float(0x7fffffff)}};
                *reinterpret_cast<float4 *>(a.maps + ((int64_t)item.slab * a.segments + item.segment) * kMaps +
                                            (threadIdx.x >> 5) * 4 + (threadIdx.x & 3)) =
                    make_float4(all.A[0], all.A[1], all.H[0], all.H[1]);
            }
        } else {
            Map2 m = run.gates(tile), pre, post, total;
            if (kBack) {
                const Map2 q = joined<true>(run.flows(tile, m));
                post = before_each<true>(q);
                total = whole<true>(q);
                pre = before_each<false>(joined<false>(m));
            } else {
                m = joined<false>(m);
                pre = before_each<false>(m);
                total = whole<false>(m);
            }
            if (item.enters) {
                const float2 v = entering(a, items[i & 3], channel);
                carry[0] = v.x;
                carry[1] = v.y;
            }
            if (!ok)  // (past a wait that ran out: no wrong state passes for a right one)
                carry[0] = carry[1] = __int_as_float(0x7fffffff);
            const bool speaks = (threadIdx.x & 31) < 4;  // one run's lanes for all
            float2 h;
            if (kBack) {
                const float *kept = c.kept(a, item, channel);
                h = make_float2(c.first ? kept[0] : 0.0f, c.second ? kept[1] : 0.0f);
                if (!ok)
                    h = make_float2(carry[0], carry[1]);
            } else {
                h = make_float2(carry[0], carry[1]);
                if (a.states && speaks) {
                    float *kept = c.kept(a, item, channel);
                    if (c.first)
                        kept[0] = h.x;
                    if (c.second)
                        kept[1] = h.y;
                }
            }
            h = make_float2(apply(pre.A[0], pre.H[0], h.x), apply(pre.A[1], pre.H[1], h.y));
            if (kBack)
                run.gradients(tile, h, make_float2(apply(post.A[0], post.H[0], carry[0]), apply(post.A[1], post.H[1], carry[1])));
            else
                run.states(tile, h);
            carry[0] = apply(total.A[0], total.H[0], carry[0]);
            carry[1] = apply(total.A[1], total.H[1], carry[1]);
            if (a.last && item.place == a.chunks - 1) {
                __syncwarp();  // (all lanes have read what entered, which may lie there)
                if (speaks && c.first)
                    a.last[item.c + channel] = carry[0];
                if (speaks && c.second)
                    a.last[item.c + channel + 1] = carry[1];
            }
            const bool out_tma = by_tma(item);
            if (out_tma)
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncthreads();
            if (out_tma) {
                if (threadIdx.x == 0) {
#pragma unroll
                    for (int k = 0; k < kOut; ++k)
#pragma unroll
                        for (int q = 0; q < kBoxes; ++q)
                            if (q * (kSlab / kBoxes) < item.width)
                                tma_store(&tma.out[k], smem_addr(stage(s, k)) + q * kBox,
                                          (int)item.d + q * (kSlab / kBoxes), (int)(c.t0 / kRun), (int)item.b);
                }
            } else {
#pragma unroll
                for (int k = 0; k < kOut; ++k) {
                    if constexpr (kTma)
                        take_out<T, kRun>(reinterpret_cast<const T *>(stage(s, k)), a.out[k], a.ot[k], a.ob[k],
                                          items[i & 3], c.t0, c.steps);
                    else
                        rows_out<T, kRun>(stage(s), a, k, items[i & 3], c.t0, c.steps);
                }
            }
            if (kTma && threadIdx.x == 0)
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        s = s_next;
    }
    if (kTma)
        asm volatile("cp.async.wait_all;" ::: "memory");
    if (kTma && kOut > 0 && threadIdx.x == 0)
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    if (!ok)
        linger();
}

// The values of a thread's two channels, all steps in registers.
template <class T, int kRun, int kArrays>
struct Column {
    T *p[kArrays][2];        // where step 0 of either channel is
    int64_t stride[kArrays];
    void *out[2][2];
    int64_t out_stride[2];
    int steps;
    bool pairs, both;        // neighbours in one access; whether there is a second
    T v[kArrays][kRun][2];

    __device__ __forceinline__ void load()
    {
#pragma unroll
        for (int q = 0; q < kArrays; ++q) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) {
                v[q][k][0] = v[q][k][1] = from_f32<T>(q == 0 ? INFINITY : 0.0f);
                if (k >= steps)
                    continue;
                const T *at = p[q][0] + k * stride[q];
                if (pairs) {
                    if constexpr (sizeof(T) == 4)
                        *reinterpret_cast<float2 *>(v[q][k]) = *reinterpret_cast<const float2 *>(at);
                    else
                        *reinterpret_cast<uint32_t *>(v[q][k]) = *reinterpret_cast<const uint32_t *>(at);
                } else {
                    v[q][k][0] = *at;
                    if (both)
                        v[q][k][1] = p[q][1][k * stride[q]];
                }
            }
        }
    }
    __device__ __forceinline__ float2 get(int array, int k) const
    {
        return make_float2(to_f32(v[array][k][0]), to_f32(v[array][k][1]));
    }
    __device__ __forceinline__ void put(int array, int k, float2 x) const
    {
        if (k >= steps)
            return;
        T *at = (T *)out[array][0] + k * out_stride[array];
        if (pairs) {
            write2(at, x);
        } else {
            *at = from_f32<T>(x.x);
            if (both)
                ((T *)out[array][1])[k * out_stride[array]] = from_f32<T>(x.y);
        }
    }
};

// Sequences of at most kRun steps: a thread takes two channels.  Eight steps of
// 4,096 x 64 16-bit values 13 us forward and 17 back (walked 39 and 53).
template <class T, bool kBack, int kRun>
__global__ __launch_bounds__(256) void brief_kernel(const Args a, bool pairs)
{
    constexpr int kArrays = kBack ? 3 : 2;
    const int64_t n = a.B * a.D, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 2;
    if (c >= n)
        return;
    Column<T, kRun, kArrays> col;
    col.pairs = pairs;
    col.both = c + 1 < n;
    col.steps = (int)a.T;
    Run<kBack, kRun> run;
    run.resets = 0;
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const int64_t cv = v && !col.both ? c : c + v, b = divide(cv, a.D), d = cv - b * a.D;
#pragma unroll
        for (int k = 0; k < kArrays; ++k) {
            col.p[k][v] = (T *)a.in[k] + b * a.ib[k] + d;
            col.stride[k] = a.it[k];
        }
#pragma unroll
        for (int k = 0; k < (kBack ? 2 : 1); ++k) {
            col.out[k][v] = (T *)a.out[k] + b * a.ob[k] + d;
            col.out_stride[k] = a.ot[k];
        }
        if (a.reset)
            for (int k = 0; k < col.steps; ++k)
                run.resets |= (a.reset[k * a.rt + b * a.rb] != 0 ? 1u : 0u) << (16 * v + k);
        const float *from = kBack ? a.states : a.first;
        (v ? s.y : s.x) = from ? from[cv] : 0.0f;
    }
    run.plain = run.resets == 0;
    col.load();
    const Map2 m = run.gates(col);
    float2 f = make_float2(0.0f, 0.0f);  // backward: what flows in from behind
    if (kBack) {
        if (a.first)
            f = make_float2(a.first[c], a.first[col.both ? c + 1 : c]);
        const Map2 q = run.flows(col, m);
        run.gradients(col, s, f);
        s = make_float2(apply(q.A[0], q.H[0], f.x), apply(q.A[1], q.H[1], f.y));
    } else {
        if (a.states) {
            a.states[c] = s.x;
            if (col.both)
                a.states[c + 1] = s.y;
        }
        run.states(col, s);
        s = make_float2(apply(m.A[0], m.H[0], s.x), apply(m.A[1], m.H[1], s.y));
    }
    if (a.last) {
        a.last[c] = s.x;
        if (col.both)
            a.last[c + 1] = s.y;
    }
}

// One step: every value once, kVec at a time.  16,384 x 256 16-bit values 14 us
// from memory, 4.1 TB/s.
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
// blocks' chunks of 16 would not fit shared memory).  Of 16-bit values 16 are
// faster (62 us against 65 on 128 steps, 98 against 135 on 4,096) but where
// half of the last of few chunks would be empty (129 steps: 151 against 113).
int run_of(int64_t T, int e)
{
    if (T <= 4 * kRuns)
        return 4;
    const int64_t rest = T % (kLongRun * kRuns);
    return T <= 8 * kRuns || e == 4 || (T < 1024 && rest > 0 && rest <= 8 * kRuns) ? 8 : kLongRun;
}
int64_t chunks_of(int64_t T, int e) { return up(T, run_of(T, e) * kRuns); }

// Blocks of channels: numbered through where the sequences lie side by side.
int64_t slabs_of(int64_t B, int64_t D, bool flat) { return flat ? up(B * D, kSlab) : B * up(D, kSlab); }

// Segments of a sequence: one where the channels fill more than a third of what
// the GPU holds (cutting reads the inputs twice), else what fills it.  Of 4,096
// steps of 16-bit values, whole and cut: 64 slabs 60 and 39 us, 100 60 and 52 (of
// 304 blocks), 120 60 and 71; of 32 bits 150 111 and 108 (of 456), 200 137 and 152.
// Few chunks are cut where there are few channels: of four, 4 slabs 10.5 and 8.8
// us (backward 16.7 and 10.6), 32 10.6 and 10.5 (16.7 and 12.6), 90 10.8 and 14.7
// (16.7 and 19.2); of two, 4 slabs 8.5 and 8.6.
int64_t segments_of(int64_t slabs, int64_t chunks, int64_t resident)
{
    if (slabs == 0 || 3 * slabs > resident || chunks <= 3 || (chunks <= 6 && 8 * slabs > resident))
        return 1;
    const int64_t most = resident / slabs, per = up(chunks, most < chunks ? most : chunks);
    return up(chunks, per);
}

int64_t resident_of(int e, bool back, int run) { return (int64_t)kSms * blocks_of(e, back, run); }

// The segments' maps, and [B D] floats for the states that enter the sequences
// where those that leave take their place.
int64_t map_bytes(int64_t slabs, int64_t segments) { return slabs * segments * kMaps * (int64_t)sizeof(Map2); }

int64_t work_bytes(int64_t T, int64_t B, int64_t D, int e)
{
    int64_t most = 0;
    for (int flat = 0; flat < 2; ++flat)
        for (int back = 0; back < 2; ++back) {
            const int64_t slabs = slabs_of(B, D, flat),
                          n = segments_of(slabs, chunks_of(T, e), resident_of(e, back, run_of(T, e)));
            const int64_t need = n > 1 ? map_bytes(slabs, n) + B * D * (int64_t)sizeof(float) : 0;
            most = need > most ? need : most;
        }
    return most;
}

// An array for TMA: channels, runs, a run's steps, sequences.
bool array_map(CUtensorMap *map, int dtype, const void *p, int64_t n, int64_t T, int run, int64_t st, int64_t B, int64_t sb)
{
    const int64_t dims[4] = {n, T / run, run, B}, strides[3] = {run * st, st, B > 1 ? sb : run * st};
    const int box[4] = {dtype == AV_F32 ? 32 : 64, kRuns, run, 1};
    return make_map(map, dtype, p, 4, dims, strides, box);
}

template <class T, bool kBack, int kRun>
cudaError_t walk(Args &a, int dtype, void *work, cudaStream_t st)
{
    constexpr int kArrays = kBack ? 3 : 2, kOut = kBack ? 2 : 1;
    const int64_t chunks = chunks_of(a.T, sizeof(T)), slabs = slabs_of(a.B, a.D, a.flat);
    const int64_t resident = resident_of(sizeof(T), kBack, kRun), segments = segments_of(slabs, chunks, resident);
    if (slabs * segments > (int64_t(1) << 30) || chunks > (int64_t(1) << 30))  // (beyond any memory)
        return cudaErrorInvalidValue;
    a.slabs = (uint32_t)slabs;
    a.chunks = (uint32_t)chunks;
    a.segments = (uint32_t)segments;
    a.per = (uint32_t)up(chunks, segments);
    a.maps = (Map2 *)work;
    if (segments > 1 && a.first && a.first == a.last) {
        // every segment begins from it, and the last may end before another begins
        float *kept = (float *)((char *)work + map_bytes(slabs, segments));
        const cudaError_t e = cudaMemcpyAsync(kept, a.first, (size_t)(a.B * a.D) * sizeof(float), cudaMemcpyDeviceToDevice, st);
        if (e != cudaSuccess)
            return e;
        a.first = kept;
    }
    const int64_t n = a.flat ? a.B * a.D : a.D, sequences = a.flat ? 1 : a.B;
    // rows of whole 16-byte pieces, a whole chunk of them at least
    bool tma = n * (int64_t)sizeof(T) % 16 == 0 && a.T >= kRun * kRuns && n < (int64_t(1) << 31) &&
               sequences < (int64_t(1) << 31);
    auto whole_pieces = [&](const void *p, int64_t t, int64_t b) {
        tma = tma && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && t * (int64_t)sizeof(T) % 16 == 0 &&
              (a.flat || b * (int64_t)sizeof(T) % 16 == 0);
    };
    auto in_words = [&](const void *p, int64_t t, int64_t b) {
        return (reinterpret_cast<uintptr_t>(p) & 3) == 0 && t % 2 == 0 && (a.flat || b % 2 == 0);
    };
    for (int k = 0; k < kArrays; ++k)
        whole_pieces(a.in[k], a.it[k], a.ib[k]);
    for (int k = 0; k < kOut; ++k) {
        whole_pieces(a.out[k], a.ot[k], a.ob[k]);
        a.words[k] = in_words(a.out[k], a.ot[k], a.ob[k]);
    }
    bool words = sizeof(T) == 2;
    for (int k = 0; k < kArrays; ++k)
        words = words && in_words(a.in[k], a.it[k], a.ib[k]);
    TensorMaps maps{};
    for (int k = 0; k < kArrays && tma; ++k)
        tma = array_map(&maps.in[k], dtype, a.in[k], n, a.T, kRun, a.it[k], sequences, a.ib[k]);
    for (int k = 0; k < kOut && tma; ++k)
        tma = array_map(&maps.out[k], dtype, a.out[k], n, a.T, kRun, a.ot[k], sequences, a.ob[k]);
    const int64_t units = slabs * segments, grid = units < resident ? units : resident;
    auto run = [&](auto kernel, int stages, int arrays, bool chained) {
        const int bytes = stages * arrays * chunk_bytes<T, kRun>(tma) + 1024;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess)
            return e;
        return launch_chained(+kernel, (unsigned)grid, kThreads, bytes, st, chained, maps, a);
    };
    auto both = [&](auto way) {
        if (segments > 1) {
            const cudaError_t e = run(walk_kernel<T, kBack, true, way.value, kRun>, stages_of(sizeof(T), kBack, true, tma), 2, false);
            if (e != cudaSuccess)
                return e;
        }
        return run(walk_kernel<T, kBack, false, way.value, kRun>, stages_of(sizeof(T), kBack, false, tma), kArrays,
                   segments > 1);
    };
    if (tma)
        return both(std::integral_constant<int, kByTma>());
    if constexpr (sizeof(T) == 2) {
        if (words)
            return both(std::integral_constant<int, kByPairs>());
    }
    return both(std::integral_constant<int, kBySingles>());
}

template <class T, bool kBack, int kRun>
cudaError_t brief(const Args &a, cudaStream_t st)
{
    // neighbours in one access: even channels are of one sequence with the next, and all arrays keep them together
    bool pairs = a.D % 2 == 0;
    auto apart = [&](const void *p, int64_t t, int64_t b) {
        pairs = pairs && (reinterpret_cast<uintptr_t>(p) & (2 * sizeof(T) - 1)) == 0 && t % 2 == 0 && b % 2 == 0;
    };
    for (int k = 0; k < (kBack ? 3 : 2); ++k)
        apart(a.in[k], a.it[k], a.ib[k]);
    for (int k = 0; k < (kBack ? 2 : 1); ++k)
        apart(a.out[k], a.ot[k], a.ob[k]);
    brief_kernel<T, kBack, kRun><<<(unsigned)up(a.B * a.D, 512), 256, 0, st>>>(a, pairs);
    return cudaGetLastError();
}

template <bool kBack>
cudaError_t launch(Args &a, int dtype, void *work, cudaStream_t st)
{
    a.flat = true;
    for (int k = 0; k < (kBack ? 3 : 2); ++k)
        a.flat = a.flat && (a.B == 1 || a.ib[k] == a.D);
    for (int k = 0; k < (kBack ? 2 : 1); ++k)
        a.flat = a.flat && (a.B == 1 || a.ob[k] == a.D);
    return with_type(dtype, [&](auto v) {
        using T = decltype(v);
        if (a.B * a.D >= kBriefChannels) {
            if (a.T <= 8)
                return a.T <= 4 ? brief<T, kBack, 4>(a, st) : brief<T, kBack, 8>(a, st);
            if constexpr (sizeof(T) == 4) {  // (16 steps of 16-bit values: 125 us against 107 walked, of 32-bit ones 50 against 114)
                if (a.T <= 16)
                    return brief<T, kBack, 16>(a, st);
            }
        }
        const int run = run_of(a.T, sizeof(T));
        if constexpr (sizeof(T) == 2) {
            if (run == kLongRun)
                return walk<T, kBack, kLongRun>(a, dtype, work, st);
        }
        return run == 4 ? walk<T, kBack, 4>(a, dtype, work, st) : walk<T, kBack, 8>(a, dtype, work, st);
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
