// C-ABI entry points of the operators around the V step: argument checks and dispatch.
#include <math.h>

#include <new>

#include "pv_ops.h"

// ---------------------------------------------------------------- scratch

pv_status pv_ops_scratch(pv_ctx *ctx, size_t bytes, void **ptr)
{
    const bool capturing = pv_capturing(ctx);
    pv_buffer &b = ctx->ops;
    if (b.ptr && b.bytes >= bytes) {
        ctx->ops_captured |= capturing;
        *ptr = b.ptr;
        return PV_OK;
    }
    if (capturing)
        return pv_fail(ctx, PV_ERR_ALLOC, "%zu bytes of scratch cannot be allocated during a capture: make a call of this size before it", bytes);
    if (b.ptr && ctx->ops_captured) {
        // graphs hold this block: it is kept until the context goes
        pv_retired *r = new (std::nothrow) pv_retired{b.ptr, ctx->retired};
        if (!r) return pv_fail(ctx, PV_ERR_ALLOC, "out of host memory");
        ctx->retired = r;
        b = pv_buffer();
        ctx->ops_captured = false;
    }
    const pv_status st = pv_ensure(ctx, b, bytes);
    *ptr = b.ptr;
    return st;
}

// ---------------------------------------------------------------- checks

static bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

static pv_status check_matrix(pv_ctx *ctx, const char *what, int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0) return pv_fail(ctx, PV_ERR_SHAPE, "%s: negative matrix shape", what);
    // rows are counted in 32 bits, with room for a tile more
    if (rows >= INT32_MAX - 1024 || cols >= INT32_MAX - 1024)
        return pv_fail(ctx, PV_ERR_SHAPE, "%s: %lld x %lld has a side of 2^31 or more", what, (long long)rows, (long long)cols);
    if (rows > 0 && pv_mx_blocks(cols) * kMxBlock >= ((int64_t)1 << 46) / rows)
        return pv_fail(ctx, PV_ERR_SHAPE, "%s: %lld x %lld is too large", what, (long long)rows, (long long)cols);
    return PV_OK;
}

static pv_status check_enums(pv_ctx *ctx, int type, int format)
{
    if (type != PV_F32 && type != PV_BF16 && type != PV_F16) return pv_fail(ctx, PV_ERR_INVALID_ARG, "unknown type %d", type);
    if (format != PV_MX_E2M1 && format != PV_MX_E4M3) return pv_fail(ctx, PV_ERR_INVALID_ARG, "unknown format %d", format);
    return PV_OK;
}

// every pointer of the list that is given is 16-byte aligned
template <class... P>
static pv_status check_aligned(pv_ctx *ctx, P... p)
{
    if ((misaligned(p) || ...)) return pv_fail(ctx, PV_ERR_INVALID_ARG, "tensor pointers must be 16-byte aligned");
    return PV_OK;
}

#define PV_CHECK(call)                             \
    do {                                           \
        const pv_status st_ = (call);              \
        if (st_ != PV_OK) return st_;              \
    } while (0)

// ---------------------------------------------------------------- microscaled formats

extern "C" pv_status pv_quantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, pv_mx_format format, pv_dtype x_type,
                                    const void *X, uint8_t *codes, uint8_t *scales)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_matrix(ctx, "X", rows, cols));
    PV_CHECK(check_enums(ctx, x_type, format));
    if (rows == 0 || cols == 0) return PV_OK;
    if (!X || !codes || !scales) return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    PV_CHECK(check_aligned(ctx, X, codes, scales));
    PV_HIP(ctx, hipSetDevice(ctx->device));
    return pv_launch_quantize_mx(ctx, rows, cols, format, x_type, X, codes, scales);
}

extern "C" pv_status pv_dequantize_mx(pv_ctx *ctx, int64_t rows, int64_t cols, pv_mx_format format, const uint8_t *codes,
                                      const uint8_t *scales, pv_dtype out_type, void *out)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_matrix(ctx, "out", rows, cols));
    PV_CHECK(check_enums(ctx, out_type, format));
    if (rows == 0 || cols == 0) return PV_OK;
    if (!out || !codes || !scales) return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    PV_CHECK(check_aligned(ctx, out, codes, scales));
    PV_HIP(ctx, hipSetDevice(ctx->device));
    return pv_launch_dequantize_mx(ctx, rows, cols, format, codes, scales, out_type, out);
}

// ---------------------------------------------------------------- product

static pv_status check_product(pv_ctx *ctx, int64_t tokens, int64_t out, int64_t in)
{
    PV_CHECK(check_matrix(ctx, "X", tokens, in));
    PV_CHECK(check_matrix(ctx, "W", out, in));
    PV_CHECK(check_matrix(ctx, "Y", tokens, out));
    return PV_OK;
}

extern "C" pv_status pv_mx_product(pv_ctx *ctx, int64_t tokens, int64_t out_features, int64_t in_features,
                                   pv_mx_format x_format, const uint8_t *x_codes, const uint8_t *x_scales,
                                   const uint8_t *w_codes, const uint8_t *w_scales, pv_dtype y_type, void *Y)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_product(ctx, tokens, out_features, in_features));
    PV_CHECK(check_enums(ctx, y_type, x_format));
    if (tokens == 0 || out_features == 0) return PV_OK;
    if (!Y) return pv_fail(ctx, PV_ERR_INVALID_ARG, "Y is NULL");
    if (in_features > 0 && (!x_codes || !x_scales || !w_codes || !w_scales))
        return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    PV_CHECK(check_aligned(ctx, Y, x_codes, x_scales, w_codes, w_scales));
    PV_HIP(ctx, hipSetDevice(ctx->device));
    if (in_features == 0) return pv_launch_zero(ctx, Y, tokens * out_features * pv_dtype_size(y_type));
    return pv_launch_mx_product(ctx, tokens, out_features, in_features, x_format, x_codes, x_scales, w_codes, w_scales,
                                y_type, Y);
}

extern "C" pv_status pv_mx_product_grads(pv_ctx *ctx, int64_t tokens, int64_t out_features, int64_t in_features,
                                         pv_mx_format x_format, const uint8_t *x_codes, const uint8_t *x_scales,
                                         const uint8_t *w_codes, const uint8_t *w_scales, const void *dY,
                                         pv_dtype dx_type, void *dX, float *dW)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_product(ctx, tokens, out_features, in_features));
    PV_CHECK(check_enums(ctx, dx_type, x_format));
    // what an empty sum leaves: zeros; what has no element: nothing (and perhaps no address)
    if (in_features == 0 || (tokens == 0 && (out_features == 0 || !dW)) || (out_features == 0 && !dX)) return PV_OK;
    if (!dX && !dW) return pv_fail(ctx, PV_ERR_INVALID_ARG, "neither gradient is asked for");
    if (tokens == 0) dX = nullptr;
    if (out_features == 0) dW = nullptr;
    if (tokens > 0 && out_features > 0 && (!dY || (dX && (!w_codes || !w_scales)) || (dW && (!x_codes || !x_scales))))
        return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    PV_CHECK(check_aligned(ctx, dX, dW, dY, x_codes, x_scales, w_codes, w_scales));
    if (dX && (dX == dY || dX == dW)) return pv_fail(ctx, PV_ERR_INVALID_ARG, "dX, dW and dY must be distinct buffers");
    if (dW && dW == dY) return pv_fail(ctx, PV_ERR_INVALID_ARG, "dX, dW and dY must be distinct buffers");
    PV_HIP(ctx, hipSetDevice(ctx->device));
    if (tokens == 0) return pv_launch_zero(ctx, dW, out_features * in_features * 4);
    if (out_features == 0) return pv_launch_zero(ctx, dX, tokens * in_features * pv_dtype_size(dx_type));
    return pv_launch_mx_product_grads(ctx, tokens, out_features, in_features, x_format, x_codes, x_scales, w_codes,
                                      w_scales, dY, dx_type, dX, dW);
}

// ---------------------------------------------------------------- norm

extern "C" pv_status pv_rms_norm(pv_ctx *ctx, int64_t rows, int64_t cols, pv_dtype type, const void *x,
                                 const void *residual, const float *weight, float eps, void *h, void *y,
                                 pv_mx_format format, uint8_t *codes, uint8_t *scales, float *rstd)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_matrix(ctx, "x", rows, cols));
    PV_CHECK(check_enums(ctx, type, format));
    if (!(eps >= 0.0f && eps < INFINITY)) return pv_fail(ctx, PV_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (rows == 0 || cols == 0) return PV_OK;
    if (!h && !y && !codes && !rstd) return pv_fail(ctx, PV_ERR_INVALID_ARG, "no output is asked for");
    if (!codes != !scales) return pv_fail(ctx, PV_ERR_INVALID_ARG, "codes and scales go together");
    if (!x || !weight) return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    if (h && h == y) return pv_fail(ctx, PV_ERR_INVALID_ARG, "h and y must be distinct buffers");
    PV_CHECK(check_aligned(ctx, x, residual, weight, h, y, codes, scales, rstd));
    PV_HIP(ctx, hipSetDevice(ctx->device));
    return pv_launch_rms_norm(ctx, rows, cols, type, x, residual, weight, eps, h, y, format, codes, scales, rstd);
}

extern "C" pv_status pv_rms_norm_backward(pv_ctx *ctx, int64_t rows, int64_t cols, pv_dtype type, const void *dy,
                                          const void *dh, const void *h, const float *weight, const float *rstd,
                                          void *dx, float *dweight)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_matrix(ctx, "dy", rows, cols));
    PV_CHECK(check_enums(ctx, type, PV_MX_E4M3));
    if (cols == 0 || (rows == 0 && !dweight)) return PV_OK;
    if (!dx && !dweight) return pv_fail(ctx, PV_ERR_INVALID_ARG, "neither gradient is asked for");
    if (rows > 0 && (!dy || !h || !weight || !rstd)) return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    PV_CHECK(check_aligned(ctx, dy, dh, h, weight, rstd, dx, dweight));
    PV_HIP(ctx, hipSetDevice(ctx->device));
    if (rows == 0) return pv_launch_zero(ctx, dweight, cols * 4);
    return pv_launch_rms_norm_backward(ctx, rows, cols, type, dy, dh, h, weight, rstd, dx, dweight);
}

// ---------------------------------------------------------------- distillation

static pv_status check_distill(pv_ctx *ctx, int64_t rows, int64_t vocab, int32_t k, int type, int64_t ld, int64_t grad_ld,
                               float temperature, const void *logits, const void *grad, const int32_t *ids, const float *top)
{
    PV_CHECK(check_matrix(ctx, "logits", rows, vocab));
    PV_CHECK(check_enums(ctx, type, PV_MX_E4M3));
    if (vocab < 1 || vocab > 1 << 20) return pv_fail(ctx, PV_ERR_SHAPE, "vocab %lld not in 1..2^20", (long long)vocab);
    if (k < 0 || k > 1024) return pv_fail(ctx, PV_ERR_INVALID_ARG, "k = %d not in 0..1024", k);
    // (its reciprocal is a normal number, and so is its square, which the loss is a part of)
    if (!(temperature >= 0x1p-126f && temperature <= 0x1p63f)) return pv_fail(ctx, PV_ERR_INVALID_ARG, "temperature not in 2^-126..2^63");
    if (ld < vocab || (grad && grad_ld < vocab)) return pv_fail(ctx, PV_ERR_SHAPE, "a row stride is below vocab");
    if (ld >= (int64_t)1 << 40 || (grad && grad_ld >= (int64_t)1 << 40) || rows * (ld >> 20) >= (int64_t)1 << 40)
        return pv_fail(ctx, PV_ERR_SHAPE, "row stride too large");
    if (rows == 0) return PV_OK;
    if (!logits || (k > 0 && (!ids || !top))) return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    if (grad == logits && grad_ld != ld) return pv_fail(ctx, PV_ERR_INVALID_ARG, "grad in place of logits needs the same row stride");
    return check_aligned(ctx, logits, grad, ids, top);
}

extern "C" pv_status pv_distill_topk(pv_ctx *ctx, int64_t rows, int64_t vocab, int32_t k, pv_dtype type, const void *logits,
                                     int64_t ld, const int32_t *teacher_ids, const float *teacher_logits,
                                     float temperature, const float *row_weight, float *loss, float *lse, void *grad,
                                     int64_t grad_ld)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_distill(ctx, rows, vocab, k, type, ld, grad_ld, temperature, logits, grad, teacher_ids, teacher_logits));
    if (rows == 0) return PV_OK;
    if (!loss) return pv_fail(ctx, PV_ERR_INVALID_ARG, "loss is NULL");
    PV_CHECK(check_aligned(ctx, row_weight, loss, lse));
    PV_HIP(ctx, hipSetDevice(ctx->device));
    return pv_launch_distill(ctx, rows, vocab, k, type, logits, ld, teacher_ids, teacher_logits, temperature, row_weight,
                             loss, lse, nullptr, grad, grad_ld);
}

extern "C" pv_status pv_distill_topk_backward(pv_ctx *ctx, int64_t rows, int64_t vocab, int32_t k, pv_dtype type,
                                              const void *logits, int64_t ld, const int32_t *teacher_ids,
                                              const float *teacher_logits, float temperature, const float *lse,
                                              const float *grad_loss, void *grad, int64_t grad_ld)
{
    if (!ctx) return PV_ERR_INVALID_ARG;
    PV_CHECK(check_distill(ctx, rows, vocab, k, type, ld, grad_ld, temperature, logits, grad, teacher_ids, teacher_logits));
    if (rows == 0) return PV_OK;
    if (!lse || !grad_loss || !grad) return pv_fail(ctx, PV_ERR_INVALID_ARG, "NULL tensor pointer");
    PV_CHECK(check_aligned(ctx, lse, grad_loss));
    PV_HIP(ctx, hipSetDevice(ctx->device));
    return pv_launch_distill(ctx, rows, vocab, k, type, logits, ld, teacher_ids, teacher_logits, temperature, grad_loss,
                             nullptr, nullptr, lse, grad, grad_ld);
}
