// k_ffn.cu -- the gated feed-forward and its gradient.
//   forward   g = x wg^T, u = x wu^T, h = act(g) u
//   backward  dg = dh u act'(g), du = dh act(g); dx = dg wg + du wu; dwg = dg^T x, dwu = du^T x
#include "policy.h"
#include "values.cuh"

namespace av {
namespace {

constexpr int kTile = 16;

// act(g) and its slope
__device__ __forceinline__ void activate(int act, float g, float &f, float &slope)
{
    if (act == AV_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        f = g * s;
        slope = s * (1.0f + g * (1.0f - s));
    } else {
        const float k = 0.7978845608028654f;  // sqrt(2 / pi)
        const float t = tanhf(k * (g + 0.044715f * g * g * g));
        f = 0.5f * g * (1.0f + t);
        slope = 0.5f * (1.0f + t) + 0.5f * g * (1.0f - t * t) * k * (1.0f + 3.0f * 0.044715f * g * g);
    }
}

// A sum of products a(i, k) b(k, j) over k, 16 x 16 results a block.
template <class A, class B>
__device__ float tile_product(int64_t i, int64_t j, int64_t n, A a, B b, float (*sa)[kTile + 1], float (*sb)[kTile + 1])
{
    float sum = 0.0f;
    for (int64_t k = 0; k < n; k += kTile) {
        __syncthreads();
        sa[threadIdx.y][threadIdx.x] = k + threadIdx.x < n ? a(i, k + threadIdx.x) : 0.0f;
        sb[threadIdx.y][threadIdx.x] = k + threadIdx.y < n ? b(k + threadIdx.y, j) : 0.0f;
        __syncthreads();
        for (int q = 0; q < kTile; ++q)
            sum += sa[threadIdx.y][q] * sb[q][threadIdx.x];
    }
    return sum;
}

// h, or with dh the projections' gradients dgu [rows][2][H].
template <class T>
__global__ void ffn_kernel(int64_t rows, int64_t D, int64_t H, int act, const T *x, int64_t xs, const T *w, T *h,
                           int64_t hs, const T *dh, int64_t dhs, T *dgu)
{
    __shared__ float sa[kTile][kTile + 1], sb[kTile][kTile + 1];
    const int64_t j = (int64_t)blockIdx.y * kTile + threadIdx.x, i = (int64_t)blockIdx.x * kTile + threadIdx.y;
    auto xv = [&](int64_t r, int64_t k) { return r < rows ? to_f32(x[r * xs + k]) : 0.0f; };
    const float g = tile_product(i, j, D, xv, [&](int64_t k, int64_t c) { return c < H ? to_f32(w[c * D + k]) : 0.0f; }, sa, sb);
    const float u = tile_product(i, j, D, xv, [&](int64_t k, int64_t c) { return c < H ? to_f32(w[(H + c) * D + k]) : 0.0f; }, sa, sb);
    if (i >= rows || j >= H)
        return;
    float f, slope;
    activate(act, g, f, slope);
    if (h)
        h[i * hs + j] = from_f32<T>(f * u);
    if (dh) {
        const float d = to_f32(dh[i * dhs + j]);
        dgu[i * 2 * H + j] = from_f32<T>(d * u * slope);
        dgu[i * 2 * H + H + j] = from_f32<T>(d * f);
    }
}

template <class T>
__global__ void ffn_dx_kernel(int64_t rows, int64_t D, int64_t H, const T *dgu, const T *w, T *dx, int64_t dxs)
{
    __shared__ float sa[kTile][kTile + 1], sb[kTile][kTile + 1];
    const int64_t j = (int64_t)blockIdx.y * kTile + threadIdx.x, i = (int64_t)blockIdx.x * kTile + threadIdx.y;
    const float v = tile_product(i, j, 2 * H, [&](int64_t r, int64_t k) { return r < rows ? to_f32(dgu[r * 2 * H + k]) : 0.0f; },
                                 [&](int64_t k, int64_t c) { return c < D ? to_f32(w[k * D + c]) : 0.0f; }, sa, sb);
    if (i < rows && j < D)
        dx[i * dxs + j] = from_f32<T>(v);
}

template <class T>
__global__ void ffn_dw_kernel(int64_t rows, int64_t D, int64_t H, const T *dgu, const T *x, int64_t xs, T *dw)
{
    __shared__ float sa[kTile][kTile + 1], sb[kTile][kTile + 1];
    const int64_t j = (int64_t)blockIdx.y * kTile + threadIdx.x, i = (int64_t)blockIdx.x * kTile + threadIdx.y;
    const float v = tile_product(i, j, rows, [&](int64_t c, int64_t r) { return c < 2 * H ? to_f32(dgu[r * 2 * H + c]) : 0.0f; },
                                 [&](int64_t r, int64_t c) { return c < D ? to_f32(x[r * xs + c]) : 0.0f; }, sa, sb);
    if (i < 2 * H && j < D)
        dw[i * D + j] = from_f32<T>(v);
}

dim3 grid_of(int64_t rows, int64_t cols) { return dim3((unsigned)((rows + kTile - 1) / kTile), (unsigned)((cols + kTile - 1) / kTile)); }

}  // namespace

int64_t ffn_work_bytes(int64_t rows, int64_t, int64_t H) { return rows * 2 * H * 2; }

cudaError_t launch_ffn(int64_t rows, int64_t D, int64_t H, int dtype, int act, const void *x, int64_t x_stride,
                       const void *w, void *h, int64_t h_stride, cudaStream_t st)
{
    with_type(dtype, [&](auto v) {
        using T = decltype(v);
        ffn_kernel<T><<<grid_of(rows, H), dim3(kTile, kTile), 0, st>>>(rows, D, H, act, (const T *)x, x_stride, (const T *)w,
                                                                (T *)h, h_stride, nullptr, 0, nullptr);
    });
    return cudaGetLastError();
}

cudaError_t launch_ffn_grad(int64_t rows, int64_t D, int64_t H, int dtype, int act, const void *dh, int64_t dh_stride,
                            const void *x, int64_t x_stride, const void *w, void *dx, int64_t dx_stride, void *dw,
                            void *work, cudaStream_t st)
{
    with_type(dtype, [&](auto v) {
        using T = decltype(v);
        ffn_kernel<T><<<grid_of(rows, H), dim3(kTile, kTile), 0, st>>>(rows, D, H, act, (const T *)x, x_stride, (const T *)w,
                                                                nullptr, 0, (const T *)dh, dh_stride, (T *)work);
        ffn_dx_kernel<T><<<grid_of(rows, D), dim3(kTile, kTile), 0, st>>>(rows, D, H, (const T *)work, (const T *)w, (T *)dx,
                                                                   dx_stride);
        ffn_dw_kernel<T><<<grid_of(2 * H, D), dim3(kTile, kTile), 0, st>>>(rows, D, H, (const T *)work, (const T *)x,
                                                                    x_stride, (T *)dw);
    });
    return cudaGetLastError();
}

}  // namespace av
