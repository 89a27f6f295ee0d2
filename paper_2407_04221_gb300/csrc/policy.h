// policy.h -- host-side launchers of the policy operators' kernels (k_norm.cu,
// k_scan.cu, k_logp.cu, k_ffn.cu).  Arguments are checked in policy.cu; a
// launcher returns what its CUDA calls returned.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "autoverse.h"

namespace av {

// A [T][B][D] array with D contiguous: strides of steps and sequences, in elements.
struct Seq {
    const void *p;
    int64_t t, b;
};
struct SeqOut {
    void *p;
    int64_t t, b;
};

cudaError_t launch_norm(int64_t rows, int n, int dtype, int param_dtype, float eps, const void *x, int64_t x_stride,
                        const void *weight, const void *bias, void *y, int64_t y_stride, float *mean, float *rstd,
                        cudaStream_t st);
cudaError_t launch_norm_grad(int64_t rows, int n, int dtype, int param_dtype, const void *dy, int64_t dy_stride,
                             const void *x, int64_t x_stride, const void *weight, const float *mean,
                             const float *rstd, void *dx, int64_t dx_stride, void *dweight, void *dbias, void *work,
                             cudaStream_t st);
int64_t norm_work_bytes(int64_t rows, int n);

cudaError_t launch_scan(int64_t T, int64_t B, int64_t D, int dtype, Seq gate, Seq value, Seq reset, const float *h0,
                        SeqOut h, float *h_last, float *states, void *work, cudaStream_t st);
cudaError_t launch_scan_grad(int64_t T, int64_t B, int64_t D, int dtype, Seq dh, Seq gate, Seq value, Seq reset,
                             const float *states, const float *dlast, SeqOut dgate, SeqOut dvalue, float *dh0,
                             void *work, cudaStream_t st);
void scan_sizes(int64_t T, int64_t B, int64_t D, int dtype, int64_t *states, int64_t *work);

struct LogpArgs {
    int64_t rows;
    int V, dtype;
    const void *logits;
    int64_t stride;
    const void *tokens;
    int token_bytes;
    const uint8_t *mask;
    int64_t mask_stride;
};
cudaError_t launch_logp(const LogpArgs &a, int top, float *logp, float *entropy, float *peak, float *logz,
                        float *top_logp, int32_t *top_index, cudaStream_t st);
cudaError_t launch_logp_grad(const LogpArgs &a, const float *dlogp, const float *dentropy, const float *peak,
                             const float *logz, const float *entropy, void *dlogits, int64_t dlogit_stride, cudaStream_t st);

cudaError_t launch_ffn(int64_t rows, int64_t D, int64_t H, int dtype, int act, const void *x, int64_t x_stride,
                       const void *w, void *h, int64_t h_stride, cudaStream_t st);
cudaError_t launch_ffn_grad(int64_t rows, int64_t D, int64_t H, int dtype, int act, const void *dh, int64_t dh_stride,
                            const void *x, int64_t x_stride, const void *w, void *dx, int64_t dx_stride, void *dw,
                            void *work, cudaStream_t st);
int64_t ffn_work_bytes(int64_t rows, int64_t D, int64_t H);

}  // namespace av
