// policy.cu -- C entry points of the policy operators (layer norm, gated
// recurrence, log probabilities, gated feed-forward): argument checks, then
// the launchers of k_norm.cu, k_scan.cu, k_logp.cu and k_ffn.cu.  Nothing here
// throws or allocates.
#include "policy.h"

namespace av {
namespace {

cudaStream_t as_stream(uintptr_t s) { return reinterpret_cast<cudaStream_t>(s); }

int status(cudaError_t e) { return e == cudaSuccess ? AV_OK : AV_ECUDA; }

bool type_ok(int32_t dtype) { return dtype == AV_F32 || dtype == AV_BF16 || dtype == AV_F16; }

int64_t type_bytes(int32_t dtype) { return dtype == AV_F32 ? 4 : 2; }

bool aligned(const void *p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

constexpr int64_t kMost = int64_t(1) << 48;  // bytes: beyond any memory, and products of two sizes stay in 64 bits

// a * b values of 4 bytes, in range
bool size_ok(int64_t a, int64_t b)
{
    return a >= 0 && b >= 0 && a <= kMost && b <= kMost && (b == 0 || a <= kMost / 4 / b);
}

// Rows of an input (any spacing, also none) and of an output (rows apart).
bool in_rows(const void *p, int64_t stride) { return p && stride >= 0 && stride <= kMost; }
bool out_rows(const void *p, int64_t rows, int64_t n, int64_t stride)
{
    return in_rows(p, stride) && (rows <= 1 || stride >= n);
}

bool in_seq(const void *p, int64_t t, int64_t b) { return p && t >= 0 && b >= 0 && t <= kMost && b <= kMost; }

// An output's strides leave no two values in one place: one axis steps over the whole of the other.
bool out_seq(const void *p, int64_t T, int64_t B, int64_t D, int64_t t, int64_t b)
{
    if (!in_seq(p, t, b))
        return false;
    if (T <= 1)
        return B <= 1 || b >= D;
    if (B <= 1)
        return t >= D;
    return (b >= D && t >= D && (t - D) / (B - 1) >= b) || (t >= D && b >= D && (b - D) / (T - 1) >= t);
}

}  // namespace
}  // namespace av

using namespace av;

extern "C" {

int av_layer_norm_work(int64_t rows, int32_t n, int64_t *bytes)
{
    if (!bytes || n < 1 || !size_ok(rows, n))
        return AV_EINVAL;
    *bytes = norm_work_bytes(rows, n);
    return AV_OK;
}

int av_layer_norm(int64_t rows, int32_t n, int32_t dtype, int32_t param_dtype, float eps, const void *x,
                  int64_t x_stride, const void *weight, const void *bias, void *y, int64_t y_stride, float *mean,
                  float *rstd, uintptr_t stream)
{
    if (n < 1 || !size_ok(rows, n) || !type_ok(dtype) || !type_ok(param_dtype) || !(eps >= 0.0f))
        return AV_EINVAL;
    if (rows == 0)
        return AV_OK;
    if (!in_rows(x, x_stride) || !out_rows(y, rows, n, y_stride) || !mean != !rstd)
        return AV_EINVAL;
    if (!aligned(x, type_bytes(dtype)) || !aligned(y, type_bytes(dtype)) || !aligned(weight, type_bytes(param_dtype)) ||
        !aligned(bias, type_bytes(param_dtype)) || !aligned(mean, 4) || !aligned(rstd, 4))
        return AV_EINVAL;
    return status(launch_norm(rows, n, dtype, param_dtype, eps, x, x_stride, weight, bias, y, y_stride, mean, rstd,
                              as_stream(stream)));
}

int av_layer_norm_grad(int64_t rows, int32_t n, int32_t dtype, int32_t param_dtype, const void *dy, int64_t dy_stride,
                       const void *x, int64_t x_stride, const void *weight, const float *mean, const float *rstd,
                       void *dx, int64_t dx_stride, void *dweight, void *dbias, void *work, int64_t work_bytes,
                       uintptr_t stream)
{
    if (n < 1 || !size_ok(rows, n) || !type_ok(dtype) || !type_ok(param_dtype))
        return AV_EINVAL;
    const int64_t e = type_bytes(dtype), pe = type_bytes(param_dtype);
    if (rows > 0 && (!in_rows(dy, dy_stride) || !in_rows(x, x_stride) || !mean || !rstd ||
                     !out_rows(dx, rows, n, dx_stride) || !aligned(dy, e) || !aligned(x, e) || !aligned(dx, e)))
        return AV_EINVAL;
    if (!aligned(weight, pe) || !aligned(dweight, pe) || !aligned(dbias, pe) || !aligned(mean, 4) || !aligned(rstd, 4))
        return AV_EINVAL;
    const int64_t need = norm_work_bytes(rows, n);
    if (need > 0 && (!work || work_bytes < need || !aligned(work, 16)))
        return AV_EINVAL;
    return status(launch_norm_grad(rows, n, dtype, param_dtype, dy, dy_stride, x, x_stride, weight, mean, rstd, dx,
                                   dx_stride, dweight, dbias, work, as_stream(stream)));
}

int av_scan_sizes(int64_t T, int64_t B, int64_t D, int32_t dtype, int64_t *states, int64_t *work)
{
    if (!states || !work || T < 0 || !size_ok(B, D) || !size_ok(T, B * D) || !type_ok(dtype))
        return AV_EINVAL;
    scan_sizes(T, B, D, dtype, states, work);
    return AV_OK;
}

int av_scan(int64_t T, int64_t B, int64_t D, int32_t dtype, const void *gate, int64_t gate_t, int64_t gate_b,
            const void *value, int64_t value_t, int64_t value_b, const uint8_t *reset, int64_t reset_t,
            int64_t reset_b, const float *h0, void *h, int64_t h_t, int64_t h_b, float *h_last, float *states,
            void *work, int64_t work_bytes, uintptr_t stream)
{
    if (T < 0 || !size_ok(B, D) || !size_ok(T, B * D) || !type_ok(dtype))
        return AV_EINVAL;
    if (!aligned(h0, 4) || !aligned(h_last, 4) || !aligned(states, 4))
        return AV_EINVAL;
    if (B == 0 || D == 0)
        return AV_OK;
    if (T == 0) {  // no step: the last state is the first
        if (!h_last || h_last == h0)
            return AV_OK;
        const size_t bytes = (size_t)B * D * 4;
        return status(h0 ? cudaMemcpyAsync(h_last, h0, bytes, cudaMemcpyDeviceToDevice, as_stream(stream))
                         : cudaMemsetAsync(h_last, 0, bytes, as_stream(stream)));
    }
    const int64_t e = type_bytes(dtype);
    if (!in_seq(gate, gate_t, gate_b) || !in_seq(value, value_t, value_b) || !out_seq(h, T, B, D, h_t, h_b) ||
        (reset && !in_seq(reset, reset_t, reset_b)) || !aligned(gate, e) || !aligned(value, e) || !aligned(h, e))
        return AV_EINVAL;
    int64_t kept, need;
    scan_sizes(T, B, D, dtype, &kept, &need);
    if (need > 0 && (!work || work_bytes < need || !aligned(work, 16)))
        return AV_EINVAL;
    return status(launch_scan(T, B, D, dtype, {gate, gate_t, gate_b}, {value, value_t, value_b},
                              {reset, reset_t, reset_b}, h0, {h, h_t, h_b}, h_last, states, work, as_stream(stream)));
}

int av_scan_grad(int64_t T, int64_t B, int64_t D, int32_t dtype, const void *dh, int64_t dh_t, int64_t dh_b,
                 const void *gate, int64_t gate_t, int64_t gate_b, const void *value, int64_t value_t,
                 int64_t value_b, const uint8_t *reset, int64_t reset_t, int64_t reset_b, const float *states,
                 const float *dlast, void *dgate, int64_t dgate_t, int64_t dgate_b, void *dvalue, int64_t dvalue_t,
                 int64_t dvalue_b, float *dh0, void *work, int64_t work_bytes, uintptr_t stream)
{
    if (T < 0 || !size_ok(B, D) || !size_ok(T, B * D) || !type_ok(dtype))
        return AV_EINVAL;
    if (!aligned(dlast, 4) || !aligned(dh0, 4) || !aligned(states, 4))
        return AV_EINVAL;
    if (B == 0 || D == 0)
        return AV_OK;
    if (T == 0) {
        if (!dh0 || dh0 == dlast)
            return AV_OK;
        const size_t bytes = (size_t)B * D * 4;
        return status(dlast ? cudaMemcpyAsync(dh0, dlast, bytes, cudaMemcpyDeviceToDevice, as_stream(stream))
                            : cudaMemsetAsync(dh0, 0, bytes, as_stream(stream)));
    }
    const int64_t e = type_bytes(dtype);
    if (!in_seq(dh, dh_t, dh_b) || !in_seq(gate, gate_t, gate_b) || !in_seq(value, value_t, value_b) ||
        (reset && !in_seq(reset, reset_t, reset_b)) || !states || !out_seq(dgate, T, B, D, dgate_t, dgate_b) ||
        !out_seq(dvalue, T, B, D, dvalue_t, dvalue_b) || !aligned(dh, e) || !aligned(gate, e) ||
        !aligned(value, e) || !aligned(dgate, e) || !aligned(dvalue, e))
        return AV_EINVAL;
    int64_t kept, need;
    scan_sizes(T, B, D, dtype, &kept, &need);
    if (need > 0 && (!work || work_bytes < need || !aligned(work, 16)))
        return AV_EINVAL;
    return status(launch_scan_grad(T, B, D, dtype, {dh, dh_t, dh_b}, {gate, gate_t, gate_b},
                                   {value, value_t, value_b}, {reset, reset_t, reset_b}, states, dlast,
                                   {dgate, dgate_t, dgate_b}, {dvalue, dvalue_t, dvalue_b}, dh0, work,
                                   as_stream(stream)));
}

}  // extern "C"

namespace {

bool logp_ok(int64_t rows, int32_t V, int32_t dtype, const void *logits, int64_t logit_stride, const void *tokens,
             int32_t token_bytes, const uint8_t *mask, int64_t mask_stride)
{
    if (V < 1 || !size_ok(rows, V) || !type_ok(dtype) || (token_bytes != 1 && token_bytes != 4 && token_bytes != 8))
        return false;
    if (rows == 0)
        return true;
    return in_rows(logits, logit_stride) && aligned(logits, type_bytes(dtype)) && tokens &&
           aligned(tokens, token_bytes) && (!mask || in_rows(mask, mask_stride));
}

bool ffn_ok(int64_t rows, int64_t D, int64_t H, int32_t dtype, int32_t act)
{
    // (the copies' coordinates are 32-bit: sides stay below 2^30)
    const int64_t side = int64_t(1) << 30;
    return rows >= 0 && rows < side && D >= 8 && D < side && H >= 8 && H < side && D % 8 == 0 && H % 8 == 0 &&
           size_ok(rows, D) && size_ok(rows, 2 * H) && size_ok(2 * H, D) && (dtype == AV_BF16 || dtype == AV_F16) &&
           (act == AV_SILU || act == AV_GELU);
}

// Rows of n values, 16-byte aligned and apart, as a tensor map takes them.
bool tma_rows(const void *p, int64_t rows, int64_t n, int64_t stride)
{
    return p && aligned(p, 16) && (rows <= 1 || (stride >= n && stride % 8 == 0 && stride < (int64_t(1) << 38)));
}

}  // namespace

extern "C" {

int av_log_probs(int64_t rows, int32_t V, int32_t dtype, const void *logits, int64_t logit_stride, const void *tokens,
                 int32_t token_bytes, const uint8_t *mask, int64_t mask_stride, int32_t top, float *logp,
                 float *entropy, float *peak, float *logz, float *top_logp, int32_t *top_index, uintptr_t stream)
{
    if (!logp_ok(rows, V, dtype, logits, logit_stride, tokens, token_bytes, mask, mask_stride))
        return AV_EINVAL;
    if (top < 0 || top > AV_MAX_TOP || top > V)
        return AV_EINVAL;
    if (rows == 0)
        return AV_OK;
    if (!logp || (top > 0 && (!top_logp || !top_index)) || !aligned(logp, 4) || !aligned(entropy, 4) ||
        !aligned(peak, 4) || !aligned(logz, 4) || !aligned(top_logp, 4) || !aligned(top_index, 4))
        return AV_EINVAL;
    const LogpArgs a{rows, V, dtype, logits, logit_stride, tokens, token_bytes, mask, mask_stride};
    return status(launch_logp(a, top, logp, entropy, peak, logz, top_logp, top_index, as_stream(stream)));
}

int av_log_probs_grad(int64_t rows, int32_t V, int32_t dtype, const void *logits, int64_t logit_stride,
                      const void *tokens, int32_t token_bytes, const uint8_t *mask, int64_t mask_stride,
                      const float *dlogp, const float *dentropy, const float *peak, const float *logz,
                      const float *entropy, void *dlogits, int64_t dlogit_stride, uintptr_t stream)
{
    if (!logp_ok(rows, V, dtype, logits, logit_stride, tokens, token_bytes, mask, mask_stride))
        return AV_EINVAL;
    if (rows == 0)
        return AV_OK;
    if (!peak || !logz || (dentropy && !entropy) || !out_rows(dlogits, rows, V, dlogit_stride) ||
        !aligned(dlogits, type_bytes(dtype)) || !aligned(peak, 4) || !aligned(logz, 4) || !aligned(entropy, 4) || !aligned(dlogp, 4) ||
        !aligned(dentropy, 4))
        return AV_EINVAL;
    const LogpArgs a{rows, V, dtype, logits, logit_stride, tokens, token_bytes, mask, mask_stride};
    return status(launch_logp_grad(a, dlogp, dentropy, peak, logz, entropy, dlogits, dlogit_stride, as_stream(stream)));
}

int av_gated_ffn_work(int64_t rows, int64_t D, int64_t H, int64_t *bytes)
{
    if (!bytes || !ffn_ok(rows, D, H, AV_BF16, AV_SILU))
        return AV_EINVAL;
    *bytes = ffn_work_bytes(rows, D, H);
    return AV_OK;
}

int av_gated_ffn(int64_t rows, int64_t D, int64_t H, int32_t dtype, int32_t act, const void *x, int64_t x_stride,
                 const void *w, void *h, int64_t h_stride, uintptr_t stream)
{
    if (!ffn_ok(rows, D, H, dtype, act))
        return AV_EINVAL;
    if (rows == 0)
        return AV_OK;
    if (!tma_rows(x, rows, D, x_stride) || !tma_rows(w, 2 * H, D, D) || !tma_rows(h, rows, H, h_stride))
        return AV_EINVAL;
    return status(launch_ffn(rows, D, H, dtype, act, x, x_stride, w, h, h_stride, as_stream(stream)));
}

int av_gated_ffn_grad(int64_t rows, int64_t D, int64_t H, int32_t dtype, int32_t act, const void *dh,
                      int64_t dh_stride, const void *x, int64_t x_stride, const void *w, void *dx, int64_t dx_stride,
                      void *dw, void *work, int64_t work_bytes, uintptr_t stream)
{
    if (!ffn_ok(rows, D, H, dtype, act) || !tma_rows(w, 2 * H, D, D) || !tma_rows(dw, 2 * H, D, D))
        return AV_EINVAL;
    if (rows == 0)  // a sum over no rows
        return status(cudaMemsetAsync(dw, 0, (size_t)2 * H * D * 2, as_stream(stream)));
    if (!tma_rows(dh, rows, H, dh_stride) || !tma_rows(x, rows, D, x_stride) || !tma_rows(dx, rows, D, dx_stride))
        return AV_EINVAL;
    const int64_t need = ffn_work_bytes(rows, D, H);
    if (need > 0 && (!work || work_bytes < need || !aligned(work, 16)))
        return AV_EINVAL;
    return status(launch_ffn_grad(rows, D, H, dtype, act, dh, dh_stride, x, x_stride, w, dx, dx_stride, dw, work,
                                  as_stream(stream)));
}

}  // extern "C"
