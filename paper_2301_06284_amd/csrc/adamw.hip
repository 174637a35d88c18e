// adamw.hip -- one AdamW step of many tensors in few launches, states in 32 or in 8 bits.
//
// A launch takes up to kPerLaunch tensors of one type combination: their pointers travel
// in the kernel's arguments, so nothing is uploaded and a captured graph holds them.  A
// workgroup takes 4096 consecutive elements of one tensor, a wave 256 of them at a time
// (4 a lane), which is one block of 8-bit states: its maximum is a reduction over one wave.
// Bound by memory.  Every product and sum is rounded on its own (no fused multiply-add), so
// that a state's code is the one that the same formula gives in any fp32 arithmetic.
#include <algorithm>
#include <cmath>
#include <vector>

#include "linear_ops.h"

namespace rgnn {

namespace {

constexpr int kPerLaunch = 48;
constexpr int kBlock = 256;               // elements of one block of 8-bit states
constexpr int kWaveSteps = 4;             // blocks a wave
constexpr int kGroup = 4 * kWaveSteps * kBlock;

struct Tensor {
    void *p;
    const void *g;
    void *m, *v;
    float *ms, *vs;
    void *copy;
    int64_t n;
};
struct StepArgs {
    Tensor t[kPerLaunch];
    int32_t first[kPerLaunch + 1];        // first workgroup of each tensor
    uint8_t vec[kPerLaunch];              // whole vectors are aligned
    uint8_t copy_type[kPerLaunch];        // rgnn_dtype
    int32_t count;
    float decay, step_size, beta1, beta2, rest1, rest2, root, eps;
    double lr, log_beta1, log_beta2;
    const int64_t *step_dev;
    const float *grad_scale;
};
static_assert(sizeof(StepArgs) <= 4096, "kernel arguments");

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

template <class P, class G, bool EIGHT, bool VEC>
__device__ __forceinline__ void update(const Tensor &t, int copy_type, const StepArgs &a, int64_t block, float step_size,
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
        int8_t cm[4];
        uint8_t cv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float q = tm > 0.0f ? rintf(127.0f * sqrtf(fabsf(m[i]) / tm)) : 0.0f;
            cm[i] = (int8_t)(int)copysignf(q, m[i]);
            const float r = tv > 0.0f ? rintf(255.0f * sqrtf(sqrtf(v[i] / tv))) : 0.0f;
            cv[i] = (uint8_t)(int)fmaxf(r, v[i] > 0.0f ? 1.0f : 0.0f);
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

template <class P, class G, bool EIGHT>
__global__ __launch_bounds__(256) void adamw_kernel(StepArgs a)
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
    const Tensor t = a.t[e];
    const bool vec = a.vec[e];
    const int64_t blocks = (t.n + kBlock - 1) / kBlock;
    const int64_t b0 = ((int64_t)((int)blockIdx.x - a.first[e]) * 4 + (threadIdx.x >> 6)) * kWaveSteps;
    for (int k = 0; k < kWaveSteps; ++k) {
        if (b0 + k >= blocks) return;
        if (vec) update<P, G, EIGHT, true>(t, a.copy_type[e], a, b0 + k, step_size, root, scale);
        else update<P, G, EIGHT, false>(t, a.copy_type[e], a, b0 + k, step_size, root, scale);
    }
}

template <class P, class G>
void launch_states(const StepArgs &a, bool eight, int64_t grid, hipStream_t s)
{
    if (eight) hipLaunchKernelGGL((adamw_kernel<P, G, true>), dim3((uint32_t)grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<P, G, false>), dim3((uint32_t)grid), dim3(256), 0, s, a);
}
template <class P>
void launch_grads(const StepArgs &a, int gd, bool eight, int64_t grid, hipStream_t s)
{
    if (gd == RGNN_F32) launch_states<P, float>(a, eight, grid, s);
    else if (gd == RGNN_BF16) launch_states<P, __bf16>(a, eight, grid, s);
    else launch_states<P, _Float16>(a, eight, grid, s);
}

bool aligned(const void *p, size_t b) { return (uintptr_t)p % b == 0; }

}  // namespace

rgnn_status launch_adamw(const rgnn_adamw_tensor_t *t, int32_t count, const rgnn_adamw_t &h, int64_t step,
                         const int64_t *step_dev, const float *grad_scale, hipStream_t s)
{
    StepArgs a{};
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
    // by type combination, in order of appearance
    std::vector<uint8_t> done(count, 0);
    bool launched = false;
    for (int32_t i = 0; i < count; ++i) {
        if (done[i] || t[i].n == 0) continue;
        int32_t k = i;
        while (k < count) {
            a.count = 0;
            int64_t grid = 0;
            for (; k < count && a.count < kPerLaunch; ++k) {
                const rgnn_adamw_tensor_t &x = t[k];
                if (done[k] || x.n == 0 || x.param_dtype != t[i].param_dtype || x.grad_dtype != t[i].grad_dtype ||
                    x.state_bits != t[i].state_bits)
                    continue;
                const int64_t groups = (x.n + kGroup - 1) / kGroup;
                if (grid + groups >= (int64_t(1) << 31) - 1) break;
                const int c = a.count++;
                const bool eight = x.state_bits == 8;
                a.t[c] = Tensor{x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, x.copy, x.n};
                a.copy_type[c] = (uint8_t)x.copy_dtype;
                a.vec[c] = aligned(x.param, 4 * dtype_bytes(x.param_dtype)) && aligned(x.grad, 4 * dtype_bytes(x.grad_dtype)) &&
                           aligned(x.m, eight ? 4 : 16) && aligned(x.v, eight ? 4 : 16) &&
                           (!x.copy || aligned(x.copy, 4 * dtype_bytes(x.copy_dtype)));
                a.first[c] = (int32_t)grid;
                grid += groups;
                done[k] = 1;
            }
            if (a.count == 0) break;
            a.first[a.count] = (int32_t)grid;
            const bool eight = t[i].state_bits == 8;
            launched = true;
            LaunchScope ls("adamw", s);
            if (t[i].param_dtype == RGNN_F32) launch_grads<float>(a, t[i].grad_dtype, eight, grid, s);
            else if (t[i].param_dtype == RGNN_BF16) launch_grads<__bf16>(a, t[i].grad_dtype, eight, grid, s);
            else launch_grads<_Float16>(a, t[i].grad_dtype, eight, grid, s);
        }
    }
    if (!launched) return RGNN_OK;
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "adamw launch");
}

}  // namespace rgnn
