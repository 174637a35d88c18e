// rows_api.cpp -- C ABI entry points of the norm, of its gradients and of dropout: argument checks, then the
// launchers.
#include <cmath>
#include <string>

#include "rows.h"

namespace rgnn {
namespace {

constexpr int64_t kMostRows = (int64_t(1) << 31) - 1;
constexpr int32_t kMostWidth = 1 << 24;

bool float_type(int32_t d) { return d == RGNN_F32 || d == RGNN_BF16 || d == RGNN_F16; }
bool on(const void *p, size_t b) { return (uintptr_t)p % b == 0; }

// The 16-bit type that a call's tensors share; bf16 where all are fp32.
struct Half {
    int type = RGNN_F32;
    bool mixed = false;
    void see(int32_t d)
    {
        if (d == RGNN_F32) return;
        mixed = mixed || (type != RGNN_F32 && type != d);
        type = d;
    }
    int of() const { return type == RGNN_F16 ? RGNN_F16 : RGNN_BF16; }
};

rgnn_status check_size(int64_t rows, int32_t cols)
{
    if (rows < 0 || cols <= 0) return fail(RGNN_EINVAL, "rows must not be negative, cols must be positive");
    if (rows >= kMostRows || cols > kMostWidth) return fail(RGNN_ERANGE, "too many rows, or cols beyond 2^24");
    return RGNN_OK;
}

rgnn_status check_matrix(const char *what, const void *p, int32_t dtype, int64_t ld, int32_t cols)
{
    const std::string w(what);
    if (!p) return fail(RGNN_EINVAL, w + " is NULL");
    if (!on(p, dtype_bytes(dtype))) return fail(RGNN_EINVAL, w + " is not on an element's boundary");
    if (ld < cols) return fail(RGNN_EINVAL, w + ": leading dimension too small");
    return RGNN_OK;
}

rgnn_status check_drop(const rgnn_dropout_t *d, DropArgs &out)
{
    if (!d) return RGNN_OK;
    if (!(d->p >= 0 && d->p <= 1)) return fail(RGNN_EINVAL, "p must lie in [0, 1]");
    if (!d->rng || !on(d->rng, 8)) return fail(RGNN_EINVAL, "rng is NULL or not on an 8-byte boundary");
    const double from = std::floor(d->p * 4294967296.0);
    out.factor = d->p < 1 ? (float)(1.0 / (1.0 - d->p)) : 0.0f;
    if (from < 1) {       // p below 2^-32: nothing is dropped, and the factor is 1
        out.factor = 1.0f;
        return RGNN_OK;
    }
    out.rng = d->rng;
    out.call = d->call;
    out.below = (uint32_t)(from - 1);
    return RGNN_OK;
}

}  // namespace
}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status rgnn_rms_norm(int32_t dtype, const void *X, int64_t rows, int64_t ldx, int32_t cols,
                                     const rgnn_dropout_t *dropout, int32_t sum_dtype, const void *residual, int64_t ldr,
                                     void *sum, int64_t lds, int32_t w_dtype, const void *weight, double eps,
                                     int32_t y_dtype, void *Y, int64_t ldy, void *scales, float *rstd, void *stream)
{
    const bool codes = dtype_eight(y_dtype);
    if (!float_type(dtype) || !float_type(sum_dtype)) return fail(RGNN_EINVAL, "X and sum must be fp32, bf16 or fp16");
    if (!codes && !float_type(y_dtype)) return fail(RGNN_EINVAL, "Y must be fp32, bf16, fp16, e4m3 or int8");
    if (weight && !float_type(w_dtype)) return fail(RGNN_EINVAL, "weight must be fp32, bf16 or fp16");
    Half half;
    half.see(dtype);
    half.see(sum_dtype);
    if (weight) half.see(w_dtype);
    if (!codes) half.see(y_dtype);
    if (half.mixed) return fail(RGNN_EINVAL, "a call's 16-bit tensors must be of one type");
    if (!std::isfinite(eps) || eps < 0) return fail(RGNN_EINVAL, "eps must be finite and not negative");
    rgnn_status st = check_size(rows, cols);
    if (st != RGNN_OK) return st;
    NormArgs a;
    if ((st = check_drop(dropout, a.drop)) != RGNN_OK) return st;
    if (rows == 0) return RGNN_OK;
    if ((st = check_matrix("X", X, dtype, ldx, cols)) != RGNN_OK) return st;
    if (residual && (st = check_matrix("residual", residual, sum_dtype, ldr, cols)) != RGNN_OK) return st;
    if (sum && (st = check_matrix("sum", sum, sum_dtype, lds, cols)) != RGNN_OK) return st;
    if (!on(weight, dtype_bytes(w_dtype))) return fail(RGNN_EINVAL, "weight is not on an element's boundary");
    if (!on(rstd, 4)) return fail(RGNN_EINVAL, "rstd is not on an element's boundary");
    if (codes) {
        if (!Y || !scales) return fail(RGNN_EINVAL, "codes or scales are NULL");
        if (!on(Y, 16) || !on(scales, 4)) return fail(RGNN_EINVAL, "codes or scales on a bad boundary");
    } else if ((st = check_matrix("Y", Y, y_dtype, ldy, cols)) != RGNN_OK) {
        return st;
    }
    a.half = half.of();
    a.x32 = dtype == RGNN_F32; a.r32 = sum_dtype == RGNN_F32; a.w32 = w_dtype == RGNN_F32;
    a.X = X; a.ldx = ldx; a.res = residual; a.ldr = ldr; a.sum = sum; a.lds = lds; a.w = weight;
    a.Y = Y; a.ldy = ldy; a.scales = scales; a.rstd = rstd;
    a.rows = rows; a.cols = cols; a.eps = eps;
    a.out = y_dtype == RGNN_F8_E4M3 ? kRowsE4m3 : y_dtype == RGNN_I8 ? kRowsInt8 : y_dtype == RGNN_F32 ? kRowsF32 : kRowsHalf;
    return launch_rms_norm(a, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_rms_norm_backward_workspace_size(int64_t rows, int32_t cols, size_t *bytes)
{
    if (!bytes) return fail(RGNN_EINVAL, "bytes is NULL");
    rgnn_status st = check_size(rows, cols);
    if (st != RGNN_OK) return st;
    *bytes = rms_norm_backward_workspace(rows, cols);
    return RGNN_OK;
}

extern "C" rgnn_status rgnn_rms_norm_backward(int32_t dy_dtype, const void *dY, int64_t rows, int64_t lddy, int32_t cols,
                                              int32_t sum_dtype, const void *sum, int64_t lds, const float *rstd,
                                              int32_t w_dtype, const void *weight, const void *d_sum, int64_t ldds,
                                              const rgnn_dropout_t *dropout, void *d_residual, int64_t lddr,
                                              int32_t dx_dtype, void *dX, int64_t lddx, int32_t dw_dtype, void *dW,
                                              void *ws, size_t ws_bytes, void *stream)
{
    if (!float_type(dy_dtype) || !float_type(sum_dtype)) return fail(RGNN_EINVAL, "dY and sum must be fp32, bf16 or fp16");
    if ((weight && !float_type(w_dtype)) || (dX && !float_type(dx_dtype)) || (dW && !float_type(dw_dtype)))
        return fail(RGNN_EINVAL, "weight, dX and dW must be fp32, bf16 or fp16");
    Half half;
    half.see(dy_dtype);
    half.see(sum_dtype);
    if (weight) half.see(w_dtype);
    if (dX) half.see(dx_dtype);
    if (dW) half.see(dw_dtype);
    if (half.mixed) return fail(RGNN_EINVAL, "a call's 16-bit tensors must be of one type");
    rgnn_status st = check_size(rows, cols);
    if (st != RGNN_OK) return st;
    NormBackwardArgs a;
    if ((st = check_drop(dropout, a.drop)) != RGNN_OK) return st;
    if (dW) {
        if (!on(dW, dtype_bytes(dw_dtype))) return fail(RGNN_EINVAL, "dW is not on an element's boundary");
        const size_t need = rms_norm_backward_workspace(rows, cols);
        if (need && (!ws || ws_bytes < need))
            return fail(RGNN_EINVAL, "workspace too small: need " + std::to_string(need) + " bytes");
        if (need && !on(ws, 16)) return fail(RGNN_EINVAL, "workspace is not on a 16-byte boundary");
    }
    if (rows > 0) {
        if ((st = check_matrix("dY", dY, dy_dtype, lddy, cols)) != RGNN_OK) return st;
        if ((st = check_matrix("sum", sum, sum_dtype, lds, cols)) != RGNN_OK) return st;
        if (!rstd || !on(rstd, 4)) return fail(RGNN_EINVAL, "rstd is NULL or not on an element's boundary");
        if (!on(weight, dtype_bytes(w_dtype))) return fail(RGNN_EINVAL, "weight is not on an element's boundary");
        if (d_sum && (st = check_matrix("d_sum", d_sum, sum_dtype, ldds, cols)) != RGNN_OK) return st;
        if (d_residual && (st = check_matrix("d_residual", d_residual, sum_dtype, lddr, cols)) != RGNN_OK) return st;
        if (dX && (st = check_matrix("dX", dX, dx_dtype, lddx, cols)) != RGNN_OK) return st;
    }
    if ((rows == 0 || (!dX && !d_residual)) && !dW) return RGNN_OK;
    a.half = half.of();
    a.dy32 = dy_dtype == RGNN_F32; a.r32 = sum_dtype == RGNN_F32; a.w32 = w_dtype == RGNN_F32;
    a.dx32 = dx_dtype == RGNN_F32; a.dw32 = dw_dtype == RGNN_F32;
    a.dY = dY; a.lddy = lddy; a.r = sum; a.ldr = lds; a.rstd = rstd; a.w = weight; a.dsum = d_sum; a.ldds = ldds;
    a.dres = d_residual; a.lddr = lddr; a.dX = dX; a.lddx = lddx; a.dW = dW; a.ws = (float *)ws;
    a.rows = rows; a.cols = cols;
    return launch_rms_norm_backward(a, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_dropout(int32_t dtype, const void *X, int64_t rows, int64_t ldx, int32_t cols,
                                    const rgnn_dropout_t *dropout, int32_t y_dtype, const void *residual, int64_t ldr,
                                    void *Y, int64_t ldy, void *stream)
{
    if (!float_type(dtype) || !float_type(y_dtype)) return fail(RGNN_EINVAL, "X and Y must be fp32, bf16 or fp16");
    Half half;
    half.see(dtype);
    half.see(y_dtype);
    if (half.mixed) return fail(RGNN_EINVAL, "a call's 16-bit tensors must be of one type");
    if (!dropout) return fail(RGNN_EINVAL, "dropout is NULL");
    rgnn_status st = check_size(rows, cols);
    if (st != RGNN_OK) return st;
    DropoutArgs a;
    if ((st = check_drop(dropout, a.drop)) != RGNN_OK) return st;
    if (rows == 0) return RGNN_OK;
    if ((st = check_matrix("X", X, dtype, ldx, cols)) != RGNN_OK) return st;
    if (residual && (st = check_matrix("residual", residual, y_dtype, ldr, cols)) != RGNN_OK) return st;
    if ((st = check_matrix("Y", Y, y_dtype, ldy, cols)) != RGNN_OK) return st;
    a.half = half.of();
    a.x32 = dtype == RGNN_F32; a.y32 = y_dtype == RGNN_F32;
    a.X = X; a.ldx = ldx; a.res = residual; a.ldr = ldr; a.Y = Y; a.ldy = ldy;
    a.rows = rows; a.cols = cols;
    return launch_dropout(a, (hipStream_t)stream);
}
