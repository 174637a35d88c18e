// adamw.hip -- one AdamW step of many tensors in few launches, states in 32 or in 8 bits.
//
// A launch takes as many tensors of one type combination as their pointers fill the 4 KB of a
// kernel's arguments, so nothing is uploaded and a captured graph holds them.  A workgroup takes up to 4096
// consecutive elements of one tensor, a wave 256 of them at a time (4 a lane), which is one block
// of 8-bit states: its maximum is a reduction over one wave.
// Bound by memory, small lists by their launches.  Measured: 201M fp32 values with bf16 gradients, bf16
// copies and 8-bit states 629 us (5.1 TB/s), 24M bf16 values in 230 tensors with fp32 states 106 us in three
// launches (5.0 TB/s), the 7 tensors of a small layer 4.8 us.  Every product and sum is rounded on its own (no fused multiply-add), so that a
// state's code is the one that the same formula gives in any fp32 arithmetic.
#include <algorithm>
#include <cmath>
#include <vector>

#include "linear_ops.h"

namespace rgnn {

namespace {

constexpr int kBlock = 256;               // elements of one block of 8-bit states

// EXTRA: with scales or copies
template <bool EXTRA>
struct StepArgs {
    static constexpr int most = EXTRA ? 56 : 86, extra = EXTRA ? most : 1;
    void *p[most];
    const void *g[most];
    void *m[most], *v[most];
    int64_t n[most];
    float *ms[extra], *vs[extra];
    void *copy[extra];
    int32_t first[most + 1];              // first workgroup of each tensor
    uint8_t flags[most];                  // 1: whole vectors are aligned; the rest: rgnn_dtype of the copy
    int32_t count, steps;                 // tensors; blocks a wave
    float decay, step_size, beta1, beta2, rest1, rest2, root, eps;
    double lr, log_beta1, log_beta2;
    const int64_t *step_dev;
    const float *grad_scale;
};
static_assert(sizeof(StepArgs<false>) <= 4096 && sizeof(StepArgs<true>) <= 4096, "kernel arguments");

struct Tensor {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    int64_t n;
};

template <class E, bool VEC>
__device__ __forceinline__ void load4(const void *base, int64_t at, int64_t n, E x[4])
{
    const E *p = (const E *)base + at;
    if (VEC && at + 4 <= n) {
        if constexpr (sizeof(E) == 4) *(i32x4 *)x = *(const i32x4 *)p;
        else if constexpr (sizeof(E) == 2) *(uint2 *)x = *(const uint2 *)p;
        else *(uint32_t *)x = *(const uint32_t *)p;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = at + i < n ? p[i] : (E)0;
}
template <class E, bool VEC>
__device__ __forceinline__ void store4(void *base, int64_t at, int64_t n, const E x[4])
{
    E *p = (E *)base + at;
    if (VEC && at + 4 <= n) {
        if constexpr (sizeof(E) == 4) *(i32x4 *)p = *(const i32x4 *)x;
        else if constexpr (sizeof(E) == 2) *(uint2 *)p = *(const uint2 *)x;
        else *(uint32_t *)p = *(const uint32_t *)x;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i < n) p[i] = x[i];
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x = fmaxf(x, __shfl_xor(x, d));
    return x;
}

template <class P, class G, bool EIGHT, bool VEC, class Args>
__device__ __forceinline__ void update(const Tensor &t, int copy_type, const Args &a, int64_t block, float step_size,
                                       float root, float scale)
{
#pragma clang fp contract(off)
    const int lane = threadIdx.x & 63;
    const int64_t at = block * kBlock + lane * 4;
    P p[4];
    G g[4];
    float m[4], v[4];
    load4<P, VEC>(t.p, at, t.n, p);
    load4<G, VEC>(t.g, at, t.n, g);
    if constexpr (EIGHT) {
        int8_t cm[4];
        uint8_t cv[4];
        load4<int8_t, VEC>(t.m, at, t.n, cm);
        load4<uint8_t, VEC>(t.v, at, t.n, cv);
        const float tm = t.ms[block], tv = t.vs[block];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = (float)cm[i] * (1.0f / 127.0f);
            m[i] = f * fabsf(f) * tm;
            float h = (float)cv[i] * (1.0f / 255.0f);
            h = h * h;
            v[i] = h * h * tv;
        }
    } else {
        load4<float, VEC>(t.m, at, t.n, m);
        load4<float, VEC>(t.v, at, t.n, v);
    }
    float np[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x = (float)g[i];
        if (a.grad_scale) x = x * scale;
        m[i] = m[i] * a.beta1 + x * a.rest1;
        v[i] = v[i] * a.beta2 + (x * x) * a.rest2;
        const float denom = sqrtf(v[i]) * root + a.eps;
        np[i] = (float)p[i] * a.decay - (m[i] / denom) * step_size;
        p[i] = (P)np[i];
    }
    store4<P, VEC>(t.p, at, t.n, p);
    if (t.copy) {
        if (copy_type == RGNN_BF16) {
            __bf16 c[4];
            for (int i = 0; i < 4; ++i) c[i] = (__bf16)np[i];
            store4<__bf16, VEC>(t.copy, at, t.n, c);
        } else if (copy_type == RGNN_F16) {
            _Float16 c[4];
            for (int i = 0; i < 4; ++i) c[i] = (_Float16)np[i];
            store4<_Float16, VEC>(t.copy, at, t.n, c);
        } else {
            store4<float, VEC>(t.copy, at, t.n, np);
        }
    }
    if constexpr (EIGHT) {
        float tm = 0.0f, tv = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            tm = fmaxf(tm, fabsf(m[i]));
            tv = fmaxf(tv, v[i]);
        }
        tm = wave_max(tm);
        tv = wave_max(tv);
        // First with one quotient a block and with roots within a unit in the last place: 127^2 / top
        // and 255^4 / top, the top scaled into [1/2, 1) and the values alike, so that neither
        // overflows.  With u = 2^-24 that is within 255 * 3.75 u of the root of the quotient, and the
        // formula in fp32 within 255 * 2.75 u: where no value is within 2e-4 of the middle
        // between two codes, the codes are the formula's.  Else (one block in six) the formula
        // itself, whose quotients and roots take three times the operations and leave memory
        // waiting (201M values: 778 us alone).
        const int em = __builtin_amdgcn_frexp_expf(tm), ev = __builtin_amdgcn_frexp_expf(tv);
        const float rm = tm > 0.0f ? 16129.0f / __builtin_amdgcn_ldexpf(tm, -em) : 0.0f;
        const float rv = tv > 0.0f ? 4228250625.0f / __builtin_amdgcn_ldexpf(tv, -ev) : 0.0f;
        float qm[4], qv[4];
        bool middle = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __builtin_amdgcn_sqrtf(__builtin_amdgcn_ldexpf(fabsf(m[i]), -em) * rm);
            const float y = __builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_ldexpf(v[i], -ev) * rv));
            qm[i] = rintf(x);
            qv[i] = rintf(y);
            middle = middle || fabsf(x - qm[i]) > 0.4998f || fabsf(y - qv[i]) > 0.4998f;
        }
        if (__ballot(middle)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                qm[i] = tm > 0.0f ? rintf(127.0f * sqrtf(fabsf(m[i]) / tm)) : 0.0f;
                qv[i] = tv > 0.0f ? rintf(255.0f * sqrtf(sqrtf(v[i] / tv))) : 0.0f;
            }
        }
        int8_t cm[4];
        uint8_t cv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cm[i] = (int8_t)(int)copysignf(qm[i], m[i]);
            cv[i] = (uint8_t)(int)fmaxf(qv[i], v[i] > 0.0f ? 1.0f : 0.0f);
        }
        store4<int8_t, VEC>(t.m, at, t.n, cm);
        store4<uint8_t, VEC>(t.v, at, t.n, cv);
        if (lane == 0) {
            t.ms[block] = tm;
            t.vs[block] = tv;
        }
    } else {
        store4<float, VEC>(t.m, at, t.n, m);
        store4<float, VEC>(t.v, at, t.n, v);
    }
}

template <class P, class G, bool EIGHT, bool EXTRA>
__global__ __launch_bounds__(256) void adamw_kernel(StepArgs<EXTRA> a)
{
    int e = 0;
    for (int k = 1; k < a.count; ++k) e += (int)blockIdx.x >= a.first[k];
    float step_size = a.step_size, root = a.root;
    if (a.step_dev) {      // the bias corrections of the step that the device counts
        const double t = (double)a.step_dev[0];
        step_size = (float)(a.lr / -expm1(t * a.log_beta1));
        root = (float)(1.0 / sqrt(-expm1(t * a.log_beta2)));
    }
    const float scale = a.grad_scale ? a.grad_scale[0] : 1.0f;
    const int flags = a.flags[e];
    const Tensor t = {a.p[e], a.g[e], a.m[e], a.v[e], EXTRA ? a.ms[e] : nullptr, EXTRA ? a.vs[e] : nullptr,
                      EXTRA ? a.copy[e] : nullptr, a.n[e]};
    const int64_t blocks = (t.n + kBlock - 1) / kBlock;
    const int64_t b0 = ((int64_t)((int)blockIdx.x - a.first[e]) * 4 + (threadIdx.x >> 6)) * a.steps;
    for (int k = 0; k < a.steps; ++k) {
        if (b0 + k >= blocks) return;
        if (flags & 1) update<P, G, EIGHT, true>(t, flags >> 1, a, b0 + k, step_size, root, scale);
        else update<P, G, EIGHT, false>(t, flags >> 1, a, b0 + k, step_size, root, scale);
    }
}

template <class P, class G>
void launch_states(const StepArgs<true> &a, bool eight, int64_t grid, hipStream_t s)
{
    if (eight) hipLaunchKernelGGL((adamw_kernel<P, G, true, true>), dim3((uint32_t)grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<P, G, false, true>), dim3((uint32_t)grid), dim3(256), 0, s, a);
}
template <class P, class G>
void launch_states(const StepArgs<false> &a, bool, int64_t grid, hipStream_t s)
{
    hipLaunchKernelGGL((adamw_kernel<P, G, false, false>), dim3((uint32_t)grid), dim3(256), 0, s, a);
}
template <class P, bool EXTRA>
void launch_grads(const StepArgs<EXTRA> &a, int gd, bool eight, int64_t grid, hipStream_t s)
{
    if (gd == RGNN_F32) launch_states<P, float>(a, eight, grid, s);
    else if (gd == RGNN_BF16) launch_states<P, __bf16>(a, eight, grid, s);
    else launch_states<P, _Float16>(a, eight, grid, s);
}

bool aligned(const void *p, size_t b) { return (uintptr_t)p % b == 0; }

// The tensors of list[begin, end), all of one type combination.
template <bool EXTRA>
void launch_some(StepArgs<EXTRA> &a, const rgnn_adamw_tensor_t *t, const std::vector<int32_t> &list, hipStream_t s)
{
    int64_t blocks = 0;
    for (int32_t i : list) blocks += (t[i].n + kBlock - 1) / kBlock;
    // up to 16 blocks a workgroup, fewer where the chip would not be full
    a.steps = (int32_t)std::min<int64_t>(4, std::max<int64_t>(1, blocks / 8192));
    size_t k = 0;
    while (k < list.size()) {
        a.count = 0;
        int64_t grid = 0;
        for (; k < list.size() && a.count < StepArgs<EXTRA>::most; ++k) {
            const rgnn_adamw_tensor_t &x = t[list[k]];
            const int64_t groups = (x.n + kBlock * 4 * a.steps - 1) / (kBlock * 4 * a.steps);
            if (grid + groups >= int64_t(1) << 24 && a.count) break;      // 2^32 threads
            const int c = a.count++;
            const bool eight = x.state_bits == 8;
            a.p[c] = x.param; a.g[c] = x.grad; a.m[c] = x.m; a.v[c] = x.v; a.n[c] = x.n;
            if constexpr (EXTRA) { a.ms[c] = x.m_scale; a.vs[c] = x.v_scale; a.copy[c] = x.copy; }
            const bool vec = aligned(x.param, 4 * dtype_bytes(x.param_dtype)) && aligned(x.grad, 4 * dtype_bytes(x.grad_dtype)) &&
                             aligned(x.m, eight ? 4 : 16) && aligned(x.v, eight ? 4 : 16) &&
                             (!x.copy || aligned(x.copy, 4 * dtype_bytes(x.copy_dtype)));
            a.flags[c] = (uint8_t)((vec ? 1 : 0) | (x.copy ? x.copy_dtype << 1 : 0));
            a.first[c] = (int32_t)grid;
            grid += groups;
        }
        a.first[a.count] = (int32_t)grid;
        const rgnn_adamw_tensor_t &x = t[list[0]];
        LaunchScope ls("adamw", s);
        if (x.param_dtype == RGNN_F32) launch_grads<float>(a, x.grad_dtype, x.state_bits == 8, grid, s);
        else if (x.param_dtype == RGNN_BF16) launch_grads<__bf16>(a, x.grad_dtype, x.state_bits == 8, grid, s);
        else launch_grads<_Float16>(a, x.grad_dtype, x.state_bits == 8, grid, s);
    }
}

template <class Args>
Args step_args(const rgnn_adamw_t &h, int64_t step, const int64_t *step_dev, const float *grad_scale)
{
    Args a{};
    const double b1 = h.beta1, b2 = h.beta2;
    // 1 - beta from the double: from beta rounded to fp32 it would be off by 1e-5 at 0.999
    a.beta1 = (float)b1; a.beta2 = (float)b2;
    a.rest1 = (float)(1.0 - b1); a.rest2 = (float)(1.0 - b2);
    a.eps = (float)h.eps; a.lr = h.lr;
    a.decay = (float)(1.0 - h.lr * h.weight_decay);
    a.log_beta1 = b1 > 0 ? std::log(b1) : -1e30; a.log_beta2 = b2 > 0 ? std::log(b2) : -1e30;
    a.step_dev = step_dev; a.grad_scale = grad_scale;
    if (!step_dev) {
        a.step_size = (float)(h.lr / -std::expm1((double)step * a.log_beta1));
        a.root = (float)(1.0 / std::sqrt(-std::expm1((double)step * a.log_beta2)));
    }
    return a;
}

}  // namespace

rgnn_status launch_adamw(const rgnn_adamw_tensor_t *t, int32_t count, const rgnn_adamw_t &h, int64_t step,
                         const int64_t *step_dev, const float *grad_scale, hipStream_t s)
{
    // by type combination: parameter, gradient, and states in 32 bits, with copies, in 8 bits
    std::vector<int32_t> lists[27];
    for (int32_t i = 0; i < count; ++i)
        if (t[i].n > 0)
            lists[t[i].param_dtype * 9 + t[i].grad_dtype * 3 + (t[i].state_bits == 8 ? 2 : t[i].copy ? 1 : 0)].push_back(i);
    bool launched = false;
    for (int l = 0; l < 27; ++l) {
        if (lists[l].empty()) continue;
        launched = true;
        if (l % 3) {
            auto a = step_args<StepArgs<true>>(h, step, step_dev, grad_scale);
            launch_some(a, t, lists[l], s);
        } else {
            auto a = step_args<StepArgs<false>>(h, step, step_dev, grad_scale);
            launch_some(a, t, lists[l], s);
        }
    }
    if (!launched) return RGNN_OK;
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "adamw launch");
}

}  // namespace rgnn
