// k_scan.cu -- the gated linear recurrence and its gradient.
//   forward   a = sigmoid(g), h_t = a k_t h_{t-1} + (1 - a) v_t
//   backward  l_t = dh_t + a_{t+1} k_{t+1} l_{t+1}; dv = (1 - a) l; dg = l (k h_{t-1} - v) a (1 - a)
#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kThreads = 128;
constexpr int kStep = 16;  // steps between kept states

// sigmoid(g) and 1 - sigmoid(g), without the cancellation of the difference
__device__ __forceinline__ void sigmoid2(float g, float &a, float &z)
{
    const float e = expf(-fabsf(g)), q = 1.0f / (1.0f + e);
    a = g >= 0.0f ? q : e * q;
    z = g >= 0.0f ? e * q : q;
}

template <class T>
__global__ void scan_kernel(int64_t Tn, int64_t B, int64_t D, const T *gate, int64_t gt, int64_t gb, const T *value,
                            int64_t vt, int64_t vb, const uint8_t *reset, int64_t rt, int64_t rb, const float *h0,
                            T *h, int64_t ht, int64_t hb, float *h_last, float *states)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= B * D)
        return;
    const int64_t b = i / D, d = i % D;
    float s = h0 ? h0[i] : 0.0f;
    for (int64_t t = 0; t < Tn; ++t) {
        if (states && t % kStep == 0)
            states[t / kStep * B * D + i] = s;
        float a, z;
        sigmoid2(to_f32(gate[t * gt + b * gb + d]), a, z);
        const bool keep = !reset || reset[t * rt + b * rb] == 0;
        s = (keep ? a * s : 0.0f) + z * to_f32(value[t * vt + b * vb + d]);
        h[t * ht + b * hb + d] = from_f32<T>(s);
    }
    if (h_last)
        h_last[i] = s;
}

template <class T>
__global__ void scan_grad_kernel(int64_t Tn, int64_t B, int64_t D, const T *dh, int64_t dht, int64_t dhb,
                                 const T *gate, int64_t gt, int64_t gb, const T *value, int64_t vt, int64_t vb,
                                 const uint8_t *reset, int64_t rt, int64_t rb, const float *states, const float *dlast,
                                 T *dgate, int64_t dgt, int64_t dgb, T *dvalue, int64_t dvt, int64_t dvb, float *dh0)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= B * D)
        return;
    const int64_t b = i / D, d = i % D;
    float l = dlast ? dlast[i] : 0.0f;
    for (int64_t c = (Tn - 1) / kStep; c >= 0; --c) {
        float before[kStep];
        float s = states[c * B * D + i];
        const int64_t t0 = c * kStep;
#pragma unroll
        for (int k = 0; k < kStep; ++k) {
            const int64_t t = t0 + k;
            if (t < Tn) {
                float a, z;
                sigmoid2(to_f32(gate[t * gt + b * gb + d]), a, z);
                before[k] = !reset || reset[t * rt + b * rb] == 0 ? s : 0.0f;
                s = a * before[k] + z * to_f32(value[t * vt + b * vb + d]);
            }
        }
#pragma unroll
        for (int k = kStep - 1; k >= 0; --k) {
            const int64_t t = t0 + k;
            if (t < Tn) {
                float a, z;
                sigmoid2(to_f32(gate[t * gt + b * gb + d]), a, z);
                l += to_f32(dh[t * dht + b * dhb + d]);
                dvalue[t * dvt + b * dvb + d] = from_f32<T>(l * z);
                dgate[t * dgt + b * dgb + d] = from_f32<T>(l * (before[k] - to_f32(value[t * vt + b * vb + d])) * a * z);
                l = !reset || reset[t * rt + b * rb] == 0 ? a * l : 0.0f;
            }
        }
    }
    if (dh0)
        dh0[i] = l;
}

}  // namespace

void scan_sizes(int64_t T, int64_t B, int64_t D, int, int64_t *states, int64_t *work)
{
    *states = (T + kStep - 1) / kStep * B * D;
    *work = 0;
}

cudaError_t launch_scan(int64_t T, int64_t B, int64_t D, int dtype, Seq gate, Seq value, Seq reset, const float *h0,
                        SeqOut h, float *h_last, float *states, void *, cudaStream_t st)
{
    with_type(dtype, [&](auto v) {
        using E = decltype(v);
        scan_kernel<E><<<(unsigned)((B * D + kThreads - 1) / kThreads), kThreads, 0, st>>>(
            T, B, D, (const E *)gate.p, gate.t, gate.b, (const E *)value.p, value.t, value.b,
            (const uint8_t *)reset.p, reset.t, reset.b, h0, (E *)h.p, h.t, h.b, h_last, states);
    });
    return cudaGetLastError();
}

cudaError_t launch_scan_grad(int64_t T, int64_t B, int64_t D, int dtype, Seq dh, Seq gate, Seq value, Seq reset,
                             const float *states, const float *dlast, SeqOut dgate, SeqOut dvalue, float *dh0, void *,
                             cudaStream_t st)
{
    with_type(dtype, [&](auto v) {
        using E = decltype(v);
        scan_grad_kernel<E><<<(unsigned)((B * D + kThreads - 1) / kThreads), kThreads, 0, st>>>(
            T, B, D, (const E *)dh.p, dh.t, dh.b, (const E *)gate.p, gate.t, gate.b, (const E *)value.p, value.t,
            value.b, (const uint8_t *)reset.p, reset.t, reset.b, states, dlast, (E *)dgate.p, dgate.t, dgate.b,
            (E *)dvalue.p, dvalue.t, dvalue.b, dh0);
    });
    return cudaGetLastError();
}

}  // namespace av
