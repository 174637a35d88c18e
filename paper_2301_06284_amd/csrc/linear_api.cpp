// linear_api.cpp -- C ABI entry points of the typed linear over device offsets (with its
// gradients and its 8-bit form) and of the AdamW step: argument checks, then the launchers.
#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "linear_ops.h"

namespace rgnn {
namespace {

constexpr int64_t kMostRows = (int64_t(1) << 31) - 1;
constexpr int32_t kMostTypes = 65535, kMostWidth = 1 << 24;

bool float_type(int32_t d) { return d == RGNN_F32 || d == RGNN_BF16 || d == RGNN_F16; }
bool on(const void *p, size_t b) { return (uintptr_t)p % b == 0; }

rgnn_status check_sizes(int64_t M, int32_t num_types, int32_t K, int32_t N)
{
    if (num_types <= 0) return fail(RGNN_EINVAL, "num_types must be positive");
    if (num_types > kMostTypes) return fail(RGNN_ERANGE, "more than 65535 types");
    if (M < 0 || K <= 0 || N <= 0) return fail(RGNN_EINVAL, "M must not be negative, K and N must be positive");
    if (M >= kMostRows) return fail(RGNN_ERANGE, "too many rows");
    if (K > kMostWidth || N > kMostWidth) return fail(RGNN_ERANGE, "K or N beyond 2^24");
    return RGNN_OK;
}

// a matrix of `rows` rows that positions 0..M-1 index, by `index` or as they are
rgnn_status check_rows(const char *what, const void *p, int32_t dtype, int64_t rows, int64_t ld, int32_t width,
                       const int32_t *index, int64_t M)
{
    const std::string w(what);
    if (!p && M > 0 && rows > 0) return fail(RGNN_EINVAL, w + " is NULL");
    if (!on(p, dtype_bytes(dtype))) return fail(RGNN_EINVAL, w + " is not on an element's boundary");
    if (rows < 0 || rows >= kMostRows) return fail(RGNN_ERANGE, w + ": bad number of rows");
    if (ld < width) return fail(RGNN_EINVAL, w + ": leading dimension too small");
    if (!index && rows < M) return fail(RGNN_EINVAL, w + " has fewer rows than there are positions");
    return RGNN_OK;
}

}  // namespace
}  // namespace rgnn

using namespace rgnn;

extern "C" rgnn_status rgnn_typed_linear(int32_t dtype, const void *X, int64_t x_rows, int64_t ldx,
                                         const int32_t *gather, const int64_t *type_ptr, int32_t num_types,
                                         int64_t M, const void *W, int32_t K, int32_t N, int32_t trans_w,
                                         int32_t y_dtype, void *Y, int64_t y_rows, int64_t ldy,
                                         const int32_t *scatter, void *stream)
{
    if (!float_type(dtype)) return fail(RGNN_EINVAL, "X and W must be fp32, bf16 or fp16");
    if (y_dtype != dtype && y_dtype != RGNN_F32) return fail(RGNN_EINVAL, "Y must be of X's type or fp32");
    if (trans_w != 0 && trans_w != 1) return fail(RGNN_EINVAL, "trans_w must be 0 or 1");
    rgnn_status st = check_sizes(M, num_types, K, N);
    if (st != RGNN_OK) return st;
    if ((st = check_rows("X", X, dtype, x_rows, ldx, K, gather, M)) != RGNN_OK) return st;
    if ((st = check_rows("Y", Y, y_dtype, y_rows, ldy, N, scatter, M)) != RGNN_OK) return st;
    if (!type_ptr || !W) return fail(RGNN_EINVAL, "NULL pointer");
    if (!on(W, dtype_bytes(dtype))) return fail(RGNN_EINVAL, "W is not on an element's boundary");
    if (M == 0) return RGNN_OK;
    LinearArgs a;
    a.dtype = dtype; a.y_dtype = y_dtype;
    a.X = X; a.x_rows = x_rows; a.ldx = ldx; a.gather = gather;
    a.type_ptr = type_ptr; a.T = num_types; a.M = M; a.W = W; a.K = K; a.N = N; a.trans_w = trans_w;
    a.Y = Y; a.y_rows = y_rows; a.ldy = ldy; a.scatter = scatter;
    return launch_typed_linear(a, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_typed_linear_wgrad_workspace_size(int32_t dtype, int64_t M, int32_t num_types, int32_t K,
                                                              int32_t N, size_t *bytes)
{
    if (!bytes) return fail(RGNN_EINVAL, "bytes is NULL");
    if (!float_type(dtype)) return fail(RGNN_EINVAL, "X and dY must be fp32, bf16 or fp16");
    rgnn_status st = check_sizes(M, num_types, K, N);
    if (st != RGNN_OK) return st;
    *bytes = wgrad_workspace(dtype, M, num_types, K, N);
    return RGNN_OK;
}

extern "C" rgnn_status rgnn_typed_linear_wgrad(int32_t dtype, const void *X, int64_t x_rows, int64_t ldx,
                                               const int32_t *gather, const void *dY, int64_t dy_rows, int64_t lddy,
                                               const int32_t *dy_gather, const int64_t *type_ptr, int32_t num_types,
                                               int64_t M, int32_t K, int32_t N, int32_t dw_dtype, void *dW, void *ws,
                                               size_t ws_bytes, void *stream)
{
    if (!float_type(dtype)) return fail(RGNN_EINVAL, "X and dY must be fp32, bf16 or fp16");
    if (dw_dtype != dtype && dw_dtype != RGNN_F32) return fail(RGNN_EINVAL, "dW must be of X's type or fp32");
    rgnn_status st = check_sizes(M, num_types, K, N);
    if (st != RGNN_OK) return st;
    if ((st = check_rows("X", X, dtype, x_rows, ldx, K, gather, M)) != RGNN_OK) return st;
    if ((st = check_rows("dY", dY, dtype, dy_rows, lddy, N, dy_gather, M)) != RGNN_OK) return st;
    if (!type_ptr || !dW) return fail(RGNN_EINVAL, "NULL pointer");
    if (!on(dW, dtype_bytes(dw_dtype))) return fail(RGNN_EINVAL, "dW is not on an element's boundary");
    const size_t need = wgrad_workspace(dtype, M, num_types, K, N);
    if (need && (!ws || ws_bytes < need))
        return fail(RGNN_EINVAL, "workspace too small: need " + std::to_string(need) + " bytes");
    if (need && !on(ws, 16)) return fail(RGNN_EINVAL, "workspace is not on a 16-byte boundary");
    WgradArgs a;
    a.dtype = dtype; a.dw_dtype = dw_dtype;
    a.X = X; a.x_rows = x_rows; a.ldx = ldx; a.gather = gather;
    a.dY = dY; a.dy_rows = dy_rows; a.lddy = lddy; a.dy_gather = dy_gather;
    a.type_ptr = type_ptr; a.T = num_types; a.M = M; a.K = K; a.N = N; a.dW = dW; a.ws = ws;
    return launch_typed_wgrad(a, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_typed_linear_select_tile(int32_t dtype, const void *X, int64_t x_rows, int64_t ldx,
                                                     const int32_t *gather, int32_t num_types, int64_t M,
                                                     const void *W, int32_t K, int32_t N, int32_t trans_w,
                                                     rgnn_tile_t *tile)
{
    if (!tile) return fail(RGNN_EINVAL, "tile is NULL");
    const bool fp8 = dtype == RGNN_F8_E4M3;
    if (!fp8 && !float_type(dtype)) return fail(RGNN_EINVAL, "X and W must be fp32, bf16, fp16 or e4m3");
    if (trans_w != (fp8 ? 1 : trans_w & 1)) return fail(RGNN_EINVAL, "trans_w must be 0 or 1, with 8 bits 1");
    rgnn_status st = check_sizes(M, num_types, K, N);
    if (st != RGNN_OK) return st;
    if ((st = check_rows("X", X, dtype, x_rows, ldx, fp8 ? fp8_width(K) : K, gather, M)) != RGNN_OK) return st;
    LinearArgs a;
    a.dtype = dtype; a.y_dtype = RGNN_F32;
    a.X = X; a.x_rows = x_rows; a.ldx = ldx; a.gather = gather;
    a.T = num_types; a.M = M; a.W = W; a.K = K; a.N = N; a.trans_w = trans_w;
    *tile = typed_linear_tile(a);
    return RGNN_OK;
}

extern "C" rgnn_status rgnn_typed_linear_wgrad_select_tile(int32_t dtype, const void *X, int64_t x_rows, int64_t ldx,
                                                           const int32_t *gather, const void *dY, int64_t dy_rows,
                                                           int64_t lddy, const int32_t *dy_gather, int32_t num_types,
                                                           int64_t M, int32_t K, int32_t N, rgnn_tile_t *tile)
{
    if (!tile) return fail(RGNN_EINVAL, "tile is NULL");
    if (!float_type(dtype)) return fail(RGNN_EINVAL, "X and dY must be fp32, bf16 or fp16");
    rgnn_status st = check_sizes(M, num_types, K, N);
    if (st != RGNN_OK) return st;
    if ((st = check_rows("X", X, dtype, x_rows, ldx, K, gather, M)) != RGNN_OK) return st;
    if ((st = check_rows("dY", dY, dtype, dy_rows, lddy, N, dy_gather, M)) != RGNN_OK) return st;
    WgradArgs a;
    a.dtype = dtype; a.dw_dtype = dtype;
    a.X = X; a.x_rows = x_rows; a.ldx = ldx; a.gather = gather;
    a.dY = dY; a.dy_rows = dy_rows; a.lddy = lddy; a.dy_gather = dy_gather;
    a.T = num_types; a.M = M; a.K = K; a.N = N;
    *tile = typed_wgrad_tile(a);
    return RGNN_OK;
}

extern "C" rgnn_status rgnn_fp8_quantize_rows(int32_t dtype, const void *X, int64_t rows, int64_t ldx, int32_t K,
                                              void *codes, uint8_t *scales, void *stream)
{
    if (!float_type(dtype)) return fail(RGNN_EINVAL, "X must be fp32, bf16 or fp16");
    if (rows < 0 || K <= 0) return fail(RGNN_EINVAL, "rows must not be negative, K must be positive");
    if (rows >= kMostRows || K > kMostWidth) return fail(RGNN_ERANGE, "too many rows, or K beyond 2^24");
    if (ldx < K) return fail(RGNN_EINVAL, "leading dimension too small");
    if (rows == 0) return RGNN_OK;
    if (!X || !codes || !scales) return fail(RGNN_EINVAL, "NULL pointer");
    if (!on(X, dtype_bytes(dtype)) || !on(codes, 16) || !on(scales, 4))
        return fail(RGNN_EINVAL, "X, codes or scales on a bad boundary");
    return launch_fp8_rows(dtype, X, rows, ldx, K, codes, scales, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_fp8_quantize_weights(int32_t dtype, const void *W, int32_t num_types, int32_t K, int32_t N,
                                                 void *codes, uint8_t *scales, void *stream)
{
    if (!float_type(dtype)) return fail(RGNN_EINVAL, "W must be fp32, bf16 or fp16");
    rgnn_status st = check_sizes(0, num_types, K, N);
    if (st != RGNN_OK) return st;
    if (!W || !codes || !scales) return fail(RGNN_EINVAL, "NULL pointer");
    if (!on(W, dtype_bytes(dtype)) || !on(codes, 16) || !on(scales, 4))
        return fail(RGNN_EINVAL, "W, codes or scales on a bad boundary");
    return launch_fp8_weights(dtype, W, num_types, K, N, codes, scales, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_typed_linear_fp8(const void *X, const uint8_t *x_scales, int64_t x_rows,
                                             const int32_t *gather, const int64_t *type_ptr, int32_t num_types,
                                             int64_t M, const void *W, const uint8_t *w_scales, int32_t K, int32_t N,
                                             int32_t y_dtype, void *Y, int64_t y_rows, int64_t ldy,
                                             const int32_t *scatter, void *stream)
{
    if (!float_type(y_dtype)) return fail(RGNN_EINVAL, "Y must be fp32, bf16 or fp16");
    rgnn_status st = check_sizes(M, num_types, K, N);
    if (st != RGNN_OK) return st;
    if ((st = check_rows("X", X, RGNN_F8_E4M3, x_rows, fp8_width(K), K, gather, M)) != RGNN_OK) return st;
    if ((st = check_rows("Y", Y, y_dtype, y_rows, ldy, N, scatter, M)) != RGNN_OK) return st;
    if (!type_ptr || !W || !w_scales || (!x_scales && M > 0 && x_rows > 0)) return fail(RGNN_EINVAL, "NULL pointer");
    if (!on(X, 16) || !on(W, 16) || !on(x_scales, 16) || !on(w_scales, 16))
        return fail(RGNN_EINVAL, "codes and scales must be on 16-byte boundaries");
    if (M == 0) return RGNN_OK;
    LinearArgs a;
    a.dtype = RGNN_F8_E4M3; a.y_dtype = y_dtype;
    a.X = X; a.x_scale = x_scales; a.x_rows = x_rows; a.ldx = fp8_width(K); a.gather = gather;
    a.type_ptr = type_ptr; a.T = num_types; a.M = M; a.W = W; a.w_scale = w_scales; a.K = K; a.N = N; a.trans_w = 1;
    a.Y = Y; a.y_rows = y_rows; a.ldy = ldy; a.scatter = scatter;
    return launch_typed_fp8(a, (hipStream_t)stream);
}

extern "C" rgnn_status rgnn_adamw_step(const rgnn_adamw_tensor_t *tensors, int32_t num_tensors,
                                       const rgnn_adamw_t *hyper, int64_t step, const int64_t *step_dev,
                                       const float *grad_scale, void *stream)
{
    if (num_tensors < 0 || (num_tensors > 0 && !tensors) || !hyper) return fail(RGNN_EINVAL, "NULL pointer or negative count");
    const rgnn_adamw_t h = *hyper;
    if (!std::isfinite(h.lr) || !std::isfinite(h.weight_decay) || !std::isfinite(h.eps) || h.eps < 0)
        return fail(RGNN_EINVAL, "lr, weight_decay and eps must be finite, eps not negative");
    if (!(h.beta1 >= 0 && h.beta1 < 1 && h.beta2 >= 0 && h.beta2 < 1)) return fail(RGNN_EINVAL, "beta1 and beta2 must lie in [0, 1)");
    if (!step_dev && step < 1) return fail(RGNN_EINVAL, "the step counts from 1");
    if (!on(step_dev, 8) || !on(grad_scale, 4)) return fail(RGNN_EINVAL, "step_dev or grad_scale on a bad boundary");
    const auto bad = [](rgnn_status st, int32_t i, const char *why) {
        return fail(st, "tensor " + std::to_string(i) + ": " + why);
    };
    bool ascending = true;
    const void *last = nullptr;
    for (int32_t i = 0; i < num_tensors; ++i) {
        const rgnn_adamw_tensor_t &t = tensors[i];
        if (t.n < 0) return bad(RGNN_EINVAL, i, "negative length");
        if (t.n > (int64_t(1) << 35)) return bad(RGNN_ERANGE, i, "too long");
        if (!float_type(t.param_dtype) || !float_type(t.grad_dtype) || (t.copy && !float_type(t.copy_dtype)))
            return bad(RGNN_EINVAL, i, "parameter, gradient and copy must be fp32, bf16 or fp16");
        if (t.state_bits != 32 && t.state_bits != 8) return bad(RGNN_EINVAL, i, "states have 32 or 8 bits");
        if (t.n == 0) continue;
        const bool eight = t.state_bits == 8;
        if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scale || !t.v_scale)))
            return bad(RGNN_EINVAL, i, "NULL pointer");
        if (!on(t.param, dtype_bytes(t.param_dtype)) || !on(t.grad, dtype_bytes(t.grad_dtype)) ||
            (t.copy && !on(t.copy, dtype_bytes(t.copy_dtype))) || (!eight && (!on(t.m, 4) || !on(t.v, 4))) ||
            (eight && (!on(t.m_scale, 4) || !on(t.v_scale, 4))))
            return bad(RGNN_EINVAL, i, "not on an element's boundary");
        ascending = ascending && last < t.param;
        last = t.param;
    }
    if (num_tensors == 0) return RGNN_OK;
    try {
        if (!ascending) {      // the same parameter twice?
            std::vector<const void *> p;
            for (int32_t i = 0; i < num_tensors; ++i)
                if (tensors[i].n) p.push_back(tensors[i].param);
            std::sort(p.begin(), p.end());
            if (std::adjacent_find(p.begin(), p.end()) != p.end())
                return fail(RGNN_EINVAL, "a parameter is named twice");
        }
        return launch_adamw(tensors, num_tensors, h, step, step_dev, grad_scale, (hipStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(RGNN_ENOMEM, "out of host memory");
    }
}
