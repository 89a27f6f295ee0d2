// k_logp.cu -- log probabilities of given tokens, entropy, top alternatives,
// and the gradient.  With m the row's largest logit and e_j = exp(x_j - m):
//   logz = log sum e,  log p_j = (x_j - m) - logz,  entropy = logz - sum e (x - m) / sum e
//   dx_j = dlogp (1[j = token] - p_j) - dentropy p_j (log p_j + entropy)
#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float no_value() { return -INFINITY; }

__device__ __forceinline__ int64_t token_of(const void *tokens, int bytes, int64_t r)
{
    return bytes == 1 ? ((const uint8_t *)tokens)[r] : bytes == 4 ? ((const int32_t *)tokens)[r]
                                                                  : ((const int64_t *)tokens)[r];
}

// (value, index) as one number, larger values first, then lower indices; NaN
// above all, both zeros alike; 0 is no entry.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t j)
{
    uint32_t u = __float_as_uint(x + 0.0f);
    u = x != x ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return (uint64_t)u << 32 | (uint32_t)~j;
}

__device__ __forceinline__ float warp_sum(float v)
{
    for (int o = 16; o; o >>= 1)
        v += __shfl_xor_sync(~0u, v, o);
    return v;
}

__device__ float block_sum(float v, float *s)
{
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        s[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
    for (int i = 0; i < kThreads / 32; ++i)
        t += s[i];
    return t;
}

__device__ float block_max(float v, float *s)
{
    for (int o = 16; o; o >>= 1)
        v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        s[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = s[0];
    for (int i = 1; i < kThreads / 32; ++i)
        t = fmaxf(t, s[i]);
    return t;
}

__device__ uint64_t block_max(uint64_t v, uint64_t *s)
{
    for (int o = 16; o; o >>= 1) {
        const uint64_t u = __shfl_xor_sync(~0u, v, o);
        v = u > v ? u : v;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        s[threadIdx.x >> 5] = v;
    __syncthreads();
    uint64_t t = s[0];
    for (int i = 1; i < kThreads / 32; ++i)
        t = s[i] > t ? s[i] : t;
    return t;
}

template <class T>
__global__ void logp_kernel(int64_t rows, int V, const T *x, int64_t xs, const void *tokens, int token_bytes,
                            const uint8_t *mask, int64_t ms, int top, float *logp, float *entropy, float *peak, float *logz,
                            float *top_logp, int32_t *top_index)
{
    __shared__ float s[kThreads / 32];
    __shared__ uint64_t sk[kThreads / 32];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + r * xs;
        const uint8_t *mr = mask ? mask + r * ms : nullptr;
        float m = no_value();
        for (int j = threadIdx.x; j < V; j += kThreads)
            if (!mr || mr[j])
                m = fmaxf(m, to_f32(xr[j]));
        m = block_max(m, s);
        float e = 0.0f, ex = 0.0f;  // sums of exp(x - m) and exp(x - m) (x - m)
        for (int j = threadIdx.x; j < V; j += kThreads) {
            const float v = to_f32(xr[j]);
            if ((mr && !mr[j]) || v == no_value())
                continue;
            const float p = expf(v - m);
            e += p;
            ex += p * (v - m);
        }
        e = block_sum(e, s);
        ex = block_sum(ex, s);
        const bool some = e != 0.0f;  // (NaN counts)
        const float z = some ? logf(e) : no_value();
        if (threadIdx.x == 0) {
            const int64_t tok = token_of(tokens, token_bytes, r);
            float lp = 0.0f;
            if (tok >= 0 && tok < V)
                lp = !some || (mr && !mr[tok]) ? no_value() : (to_f32(xr[tok]) - m) - z;
            logp[r] = lp;
            if (entropy)
                entropy[r] = some ? z - ex / e : 0.0f;
            if (peak)
                peak[r] = m;
            if (logz)
                logz[r] = z;
        }
        uint64_t last = ~0ull;
        for (int k = 0; k < top; ++k) {
            uint64_t best = 0;
            for (int j = threadIdx.x; j < V; j += kThreads) {
                const float v = to_f32(xr[j]);
                if ((mr && !mr[j]) || v == no_value())
                    continue;
                const uint64_t key = rank_key(v, j);
                if (key < last && key > best)
                    best = key;
            }
            best = block_max(best, sk);
            last = best;
            if (threadIdx.x == 0) {
                const int j = best ? (int)~(uint32_t)best : -1;
                top_index[r * top + k] = j;
                top_logp[r * top + k] = best ? (to_f32(xr[j]) - m) - z : no_value();
            }
        }
    }
}

template <class T>
__global__ void logp_grad_kernel(int64_t rows, int V, const T *x, int64_t xs, const void *tokens, int token_bytes,
                                 const uint8_t *mask, int64_t ms, const float *dlogp, const float *dentropy,
                                 const float *peak, const float *logz, const float *entropy, T *dx, int64_t dxs)
{
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float m = peak[r], z = logz[r], de = dentropy ? dentropy[r] : 0.0f, h = dentropy ? entropy[r] : 0.0f;
        const int64_t tok = token_of(tokens, token_bytes, r);
        const float dl = dlogp && tok >= 0 && tok < V ? dlogp[r] : 0.0f;
        for (int j = threadIdx.x; j < V; j += kThreads) {
            float g = 0.0f;
            if (z != no_value() && !(mask && !mask[r * ms + j])) {
                const float lp = (to_f32(x[r * xs + j]) - m) - z, p = expf(lp);
                g = (j == tok ? dl : 0.0f) - p * dl - (p == 0.0f ? 0.0f : de * p * (lp + h));
            }
            dx[r * dxs + j] = from_f32<T>(g);
        }
    }
}

unsigned grid_of(int64_t rows) { return (unsigned)(rows < 152 * 8 ? rows : 152 * 8); }

}  // namespace

cudaError_t launch_logp(const LogpArgs &a, int top, float *logp, float *entropy, float *peak, float *logz,
                        float *top_logp, int32_t *top_index, cudaStream_t st)
{
    with_type(a.dtype, [&](auto v) {
        using T = decltype(v);
        logp_kernel<T><<<grid_of(a.rows), kThreads, 0, st>>>(a.rows, a.V, (const T *)a.logits, a.stride, a.tokens,
                                                             a.token_bytes, a.mask, a.mask_stride, top, logp, entropy, peak, logz, top_logp, top_index);
    });
    return cudaGetLastError();
}

cudaError_t launch_logp_grad(const LogpArgs &a, const float *dlogp, const float *dentropy, const float *peak,
                             const float *logz, const float *entropy, void *dlogits, int64_t dlogit_stride, cudaStream_t st)
{
    with_type(a.dtype, [&](auto v) {
        using T = decltype(v);
        logp_grad_kernel<T><<<grid_of(a.rows), kThreads, 0, st>>>(a.rows, a.V, (const T *)a.logits, a.stride, a.tokens,
                                                                  a.token_bytes, a.mask, a.mask_stride, dlogp,
                                                                  dentropy, peak, logz, entropy, (T *)dlogits, dlogit_stride);
    });
    return cudaGetLastError();
}

}  // namespace av
