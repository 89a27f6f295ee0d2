// k_norm.cu -- layer norm of rows and its gradient.
//   forward   mean, var of a row, y = (x - mean) rstd w + b
//   backward  d = dy w; dx = rstd (d - mean(d) - xh mean(d xh)); dw = sum_rows dy xh; db = sum_rows dy
#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kThreads = 256;

// Sum over the block, in every thread; the same order whatever the timing.
__device__ float block_sum(float v, float *s)
{
    for (int o = 16; o; o >>= 1)
        v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        s[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
    for (int i = 0; i < (int)blockDim.x / 32; ++i)
        t += s[i];
    return t;
}

template <class T, class P>
__global__ void norm_kernel(int64_t rows, int n, float eps, const T *x, int64_t xs, const P *w, const P *b, T *y,
                            int64_t ys, float *mean, float *rstd)
{
    __shared__ float s[kThreads / 32];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + r * xs;
        float v = 0.0f;
        for (int i = threadIdx.x; i < n; i += kThreads)
            v += to_f32(xr[i]);
        const float m = block_sum(v, s) / n;
        v = 0.0f;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float c = to_f32(xr[i]) - m;
            v += c * c;
        }
        const float q = 1.0f / sqrtf(block_sum(v, s) / n + eps);
        for (int i = threadIdx.x; i < n; i += kThreads)
            y[r * ys + i] = from_f32<T>((to_f32(xr[i]) - m) * q * (w ? to_f32(w[i]) : 1.0f) + (b ? to_f32(b[i]) : 0.0f));
        if (mean && threadIdx.x == 0) {
            mean[r] = m;
            rstd[r] = q;
        }
    }
}

template <class T, class P>
__global__ void norm_dx_kernel(int64_t rows, int n, const T *dy, int64_t dys, const T *x, int64_t xs, const P *w,
                               const float *mean, const float *rstd, T *dx, int64_t dxs)
{
    __shared__ float s[kThreads / 32];
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
        const float m = mean[r], q = rstd[r];
        float a = 0.0f, c = 0.0f;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float d = to_f32(dy[r * dys + i]) * (w ? to_f32(w[i]) : 1.0f);
            a += d;
            c += d * (to_f32(x[r * xs + i]) - m) * q;
        }
        a = block_sum(a, s) / n;
        c = block_sum(c, s) / n;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float d = to_f32(dy[r * dys + i]) * (w ? to_f32(w[i]) : 1.0f);
            const float xh = (to_f32(x[r * xs + i]) - m) * q;
            dx[r * dxs + i] = from_f32<T>(q * (d - a - xh * c));
        }
    }
}

// A block takes 32 columns, its warps rows in turn.
template <class T, class P>
__global__ void norm_dw_kernel(int64_t rows, int n, const T *dy, int64_t dys, const T *x, int64_t xs,
                               const float *mean, const float *rstd, P *dw, P *db)
{
    __shared__ float s[2][kThreads / 32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    float a = 0.0f, c = 0.0f;
    if (i < n)
        for (int64_t r = warp; r < rows; r += kThreads / 32) {
            const float d = to_f32(dy[r * dys + i]);
            a += d * (to_f32(x[r * xs + i]) - mean[r]) * rstd[r];
            c += d;
        }
    s[0][warp][lane] = a;
    s[1][warp][lane] = c;
    __syncthreads();
    if (warp != 0 || i >= n)
        return;
    for (int k = 1; k < kThreads / 32; ++k) {
        a += s[0][k][lane];
        c += s[1][k][lane];
    }
    if (dw)
        dw[i] = from_f32<P>(a);
    if (db)
        db[i] = from_f32<P>(c);
}

unsigned grid_of(int64_t rows) { return (unsigned)(rows < 152 * 8 ? rows : 152 * 8); }

}  // namespace

int64_t norm_work_bytes(int64_t, int) { return 0; }

cudaError_t launch_norm(int64_t rows, int n, int dtype, int param_dtype, float eps, const void *x, int64_t x_stride,
                        const void *weight, const void *bias, void *y, int64_t y_stride, float *mean, float *rstd,
                        cudaStream_t st)
{
    with_type(dtype, [&](auto t) {
        with_type(param_dtype, [&](auto p) {
            using T = decltype(t);
            using P = decltype(p);
            norm_kernel<T, P><<<grid_of(rows), kThreads, 0, st>>>(rows, n, eps, (const T *)x, x_stride,
                                                                  (const P *)weight, (const P *)bias, (T *)y, y_stride,
                                                                  mean, rstd);
        });
    });
    return cudaGetLastError();
}

cudaError_t launch_norm_grad(int64_t rows, int n, int dtype, int param_dtype, const void *dy, int64_t dy_stride,
                             const void *x, int64_t x_stride, const void *weight, const float *mean,
                             const float *rstd, void *dx, int64_t dx_stride, void *dweight, void *dbias, void *,
                             cudaStream_t st)
{
    with_type(dtype, [&](auto t) {
        with_type(param_dtype, [&](auto p) {
            using T = decltype(t);
            using P = decltype(p);
            if (rows > 0)
                norm_dx_kernel<T, P><<<grid_of(rows), kThreads, 0, st>>>(rows, n, (const T *)dy, dy_stride,
                                                                         (const T *)x, x_stride, (const P *)weight,
                                                                         mean, rstd, (T *)dx, dx_stride);
            if (dweight || dbias)
                norm_dw_kernel<T, P><<<(n + 31) / 32, kThreads, 0, st>>>(rows, n, (const T *)dy, dy_stride,
                                                                         (const T *)x, x_stride, mean, rstd,
                                                                         (P *)dweight, (P *)dbias);
        });
    });
    return cudaGetLastError();
}

}  // namespace av
