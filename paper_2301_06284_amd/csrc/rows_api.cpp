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
    const auto bad = [what](const char *why) { return fail(RGNN_EINVAL, std::string(what) + why); };
    if (!p) return bad(" is NULL");
    if (!on(p, dtype_bytes(dtype))) return bad(" is not on an element's boundary");
    if (ld < cols) return bad(": leading dimension too small");
    return RGNN_OK;
}

// D as the kernels take it; nothing without rng.
rgnn_status check_drop(const rgnn_dropout_t &d, DropArgs &out)
{
    if (!d.rng) return RGNN_OK;
    if (!(d.p >= 0 && d.p <= 1)) return fail(RGNN_EINVAL, "p must lie in [0, 1]");
    if (!on(d.rng, 8)) return fail(RGNN_EINVAL, "rng is not on an 8-byte boundary");
    const double from = std::floor(d.p * 4294967296.0);
    if (from < 1) return RGNN_OK;       // p below 2^-32: nothing is dropped, and the factor is 1
    out.factor = d.p < 1 ? (float)(1.0 / (1.0 - d.p)) : 0.0f;
    out.rng = d.rng;
    out.call = d.call;
    out.below = (uint32_t)(from - 1);
    return RGNN_OK;
}

}  // namespace
}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status rgnn_rms_norm(const rgnn_rms_norm_t *args, void *stream)
{
    if (!args) return fail(RGNN_EINVAL, "args is NULL");
    const rgnn_rms_norm_t &p = *args;
    const int32_t dtype = p.dtype, sum_dtype = p.sum_dtype, w_dtype = p.w_dtype, y_dtype = p.y_dtype, cols = p.cols;
    const int64_t rows = p.rows;
    const bool codes = dtype_eight(y_dtype);
    if (!float_type(dtype) || !float_type(sum_dtype)) return fail(RGNN_EINVAL, "X and sum must be fp32, bf16 or fp16");
    if (!codes && !float_type(y_dtype)) return fail(RGNN_EINVAL, "Y must be fp32, bf16, fp16, e4m3 or int8");
    if (p.weight && !float_type(w_dtype)) return fail(RGNN_EINVAL, "weight must be fp32, bf16 or fp16");
    Half half;
    half.see(dtype);
    half.see(sum_dtype);
    if (p.weight) half.see(w_dtype);
    if (!codes) half.see(y_dtype);
    if (half.mixed) return fail(RGNN_EINVAL, "a call's 16-bit tensors must be of one type");
    if (!std::isfinite(p.eps) || p.eps < 0) return fail(RGNN_EINVAL, "eps must be finite and not negative");
    rgnn_status st = check_size(rows, cols);
    if (st != RGNN_OK) return st;
    NormArgs a;
    if ((st = check_drop(p.dropout, a.drop)) != RGNN_OK) return st;
    if (rows == 0) return RGNN_OK;
    if ((st = check_matrix("X", p.X, dtype, p.ldx, cols)) != RGNN_OK) return st;
    if (p.residual && (st = check_matrix("residual", p.residual, sum_dtype, p.ldr, cols)) != RGNN_OK) return st;
    if (p.sum && (st = check_matrix("sum", p.sum, sum_dtype, p.lds, cols)) != RGNN_OK) return st;
    if (!on(p.weight, dtype_bytes(w_dtype))) return fail(RGNN_EINVAL, "weight is not on an element's boundary");
    if (!on(p.rstd, 4)) return fail(RGNN_EINVAL, "rstd is not on an element's boundary");
    if (codes) {
        if (!p.Y || !p.scales) return fail(RGNN_EINVAL, "codes or scales are NULL");
        if (!on(p.Y, 16) || !on(p.scales, 4)) return fail(RGNN_EINVAL, "codes or scales on a bad boundary");
    } else if ((st = check_matrix("Y", p.Y, y_dtype, p.ldy, cols)) != RGNN_OK) {
        return st;
    }
    a.half = half.of();
    a.x32 = dtype == RGNN_F32; a.r32 = sum_dtype == RGNN_F32; a.w32 = w_dtype == RGNN_F32;
    a.X = p.X; a.ldx = p.ldx; a.res = p.residual; a.ldr = p.ldr; a.sum = p.sum; a.lds = p.lds; a.w = p.weight;
    a.Y = p.Y; a.ldy = p.ldy; a.scales = p.scales; a.rstd = p.rstd;
    a.rows = rows; a.cols = cols; a.eps = p.eps;
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

extern "C" rgnn_status rgnn_rms_norm_backward(const rgnn_rms_norm_backward_t *args, void *stream)
{
    if (!args) return fail(RGNN_EINVAL, "args is NULL");
    const rgnn_rms_norm_backward_t &p = *args;
    const int32_t dy_dtype = p.dy_dtype, sum_dtype = p.sum_dtype, w_dtype = p.w_dtype, dx_dtype = p.dx_dtype, dw_dtype = p.dw_dtype;
    const int32_t cols = p.cols;
    const int64_t rows = p.rows;
    if (!float_type(dy_dtype) || !float_type(sum_dtype)) return fail(RGNN_EINVAL, "dY and sum must be fp32, bf16 or fp16");
    if ((p.weight && !float_type(w_dtype)) || (p.dX && !float_type(dx_dtype)) || (p.dW && !float_type(dw_dtype)))
        return fail(RGNN_EINVAL, "weight, dX and dW must be fp32, bf16 or fp16");
    Half half;
    half.see(dy_dtype);
    half.see(sum_dtype);
    if (p.weight) half.see(w_dtype);
    if (p.dX) half.see(dx_dtype);
    if (p.dW) half.see(dw_dtype);
    if (half.mixed) return fail(RGNN_EINVAL, "a call's 16-bit tensors must be of one type");
    rgnn_status st = check_size(rows, cols);
    if (st != RGNN_OK) return st;
    NormBackwardArgs a;
    if ((st = check_drop(p.dropout, a.drop)) != RGNN_OK) return st;
    if (p.dW) {
        if (!on(p.dW, dtype_bytes(dw_dtype))) return fail(RGNN_EINVAL, "dW is not on an element's boundary");
        const size_t need = rms_norm_backward_workspace(rows, cols);
        if (need && (!p.ws || p.ws_bytes < need))
            return fail(RGNN_EINVAL, "workspace too small: need " + std::to_string(need) + " bytes");
        if (need && !on(p.ws, 16)) return fail(RGNN_EINVAL, "workspace is not on a 16-byte boundary");
    }
    if (rows > 0) {
        if ((st = check_matrix("dY", p.dY, dy_dtype, p.lddy, cols)) != RGNN_OK) return st;
        if ((st = check_matrix("sum", p.sum, sum_dtype, p.lds, cols)) != RGNN_OK) return st;
        if (!p.rstd || !on(p.rstd, 4)) return fail(RGNN_EINVAL, "rstd is NULL or not on an element's boundary");
        if (!on(p.weight, dtype_bytes(w_dtype))) return fail(RGNN_EINVAL, "weight is not on an element's boundary");
        if (p.d_sum && (st = check_matrix("d_sum", p.d_sum, sum_dtype, p.ldds, cols)) != RGNN_OK) return st;
        if (p.d_residual && (st = check_matrix("d_residual", p.d_residual, sum_dtype, p.lddr, cols)) != RGNN_OK) return st;
        if (p.dX && (st = check_matrix("dX", p.dX, dx_dtype, p.lddx, cols)) != RGNN_OK) return st;
    }
    if ((rows == 0 || (!p.dX && !p.d_residual)) && !p.dW) return RGNN_OK;
    a.half = half.of();
    a.dy32 = dy_dtype == RGNN_F32; a.r32 = sum_dtype == RGNN_F32; a.w32 = w_dtype == RGNN_F32;
    a.dx32 = dx_dtype == RGNN_F32; a.dw32 = dw_dtype == RGNN_F32;
    a.dY = p.dY; a.lddy = p.lddy; a.r = p.sum; a.ldr = p.lds; a.rstd = p.rstd; a.w = p.weight; a.dsum = p.d_sum; a.ldds = p.ldds;
    a.dres = p.d_residual; a.lddr = p.lddr; a.dX = p.dX; a.lddx = p.lddx; a.dW = p.dW; a.ws = (float *)p.ws;
    a.rows = rows; a.cols = cols;
    return launch_rms_norm_backward(a, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_dropout(const rgnn_dropout_rows_t *args, void *stream)
{
    if (!args) return fail(RGNN_EINVAL, "args is NULL");
    const rgnn_dropout_rows_t &p = *args;
    const int32_t dtype = p.dtype, y_dtype = p.y_dtype, cols = p.cols;
    const int64_t rows = p.rows;
    if (!float_type(dtype) || !float_type(y_dtype)) return fail(RGNN_EINVAL, "X and Y must be fp32, bf16 or fp16");
    Half half;
    half.see(dtype);
    half.see(y_dtype);
    if (half.mixed) return fail(RGNN_EINVAL, "a call's 16-bit tensors must be of one type");
    rgnn_status st = check_size(rows, cols);
    if (st != RGNN_OK) return st;
    DropoutArgs a;
    if ((st = check_drop(p.dropout, a.drop)) != RGNN_OK) return st;
    if (rows == 0) return RGNN_OK;
    if ((st = check_matrix("X", p.X, dtype, p.ldx, cols)) != RGNN_OK) return st;
    if (p.residual && (st = check_matrix("residual", p.residual, y_dtype, p.ldr, cols)) != RGNN_OK) return st;
    if ((st = check_matrix("Y", p.Y, y_dtype, p.ldy, cols)) != RGNN_OK) return st;
    a.half = half.of();
    a.x32 = dtype == RGNN_F32; a.y32 = y_dtype == RGNN_F32;
    a.X = p.X; a.ldx = p.ldx; a.res = p.residual; a.ldr = p.ldr; a.Y = p.Y; a.ldy = p.ldy;
    a.rows = rows; a.cols = cols;
    return launch_dropout(a, (hipStream_t)stream);
}
