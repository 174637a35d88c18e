// rows.h -- what the kernels over rows share (norm, its backward, dropout, 8-bit integers): vectors of eight
// columns from any address, sums and maxima over the lanes of a row, the generator of dropout's
// numbers, rows of 8-bit codes.
#pragma once

#include "linear_ops.h"
#include "wave_ops.h"

namespace rgnn {

// What decides a dropped value, as the kernels take it.  rng NULL: nothing is dropped.
struct DropArgs {
    const int64_t *rng = nullptr;    // device: seed, offset
    int64_t call = 0;
    uint32_t below = 0;              // numbers up to this one are dropped
    float factor = 1.0f;             // what is kept times this
};

// The output of a norm.
enum RowsOut : int { kRowsHalf = 0, kRowsF32 = 1, kRowsE4m3 = 2, kRowsInt8 = 3 };

struct NormArgs {
    int half = 0;                    // rgnn_dtype of the call's 16-bit type
    bool x32 = false, r32 = false, w32 = false;    // fp32 X, residual and sum, weight
    const void *X = nullptr;     int64_t ldx = 0;
    const void *res = nullptr;   int64_t ldr = 0;
    void *sum = nullptr;         int64_t lds = 0;
    const void *w = nullptr;
    void *Y = nullptr;           int64_t ldy = 0;
    void *scales = nullptr;
    float *rstd = nullptr;
    int64_t rows = 0;
    int32_t cols = 0;
    int out = kRowsHalf;
    double eps = 0;
    DropArgs drop;
};

struct NormBackwardArgs {
    int half = 0;
    bool dy32 = false, r32 = false, w32 = false, dx32 = false, dw32 = false;
    const void *dY = nullptr;    int64_t lddy = 0;
    const void *r = nullptr;     int64_t ldr = 0;
    const float *rstd = nullptr;
    const void *w = nullptr;
    const void *dsum = nullptr;  int64_t ldds = 0;
    void *dres = nullptr;        int64_t lddr = 0;
    void *dX = nullptr;          int64_t lddx = 0;
    void *dW = nullptr;
    float *ws = nullptr;
    int64_t rows = 0;
    int32_t cols = 0;
    DropArgs drop;
};

struct DropoutArgs {
    int half = 0;
    bool x32 = false, y32 = false;
    const void *X = nullptr;     int64_t ldx = 0;
    const void *res = nullptr;   int64_t ldr = 0;
    void *Y = nullptr;           int64_t ldy = 0;
    int64_t rows = 0;
    int32_t cols = 0;
    DropArgs drop;
};

rgnn_status launch_rms_norm(const NormArgs &a, hipStream_t s);
rgnn_status launch_rms_norm_backward(const NormBackwardArgs &a, hipStream_t s);
size_t rms_norm_backward_workspace(int64_t rows, int32_t cols);
rgnn_status launch_dropout(const DropoutArgs &a, hipStream_t s);

#ifdef __HIPCC__

// ---------------------------------------------------------------- eight columns

// Eight values side by side, or the first `left` of them and zeros, from any address of an element: a vector
// load takes any address, at full speed where it is a multiple of its size.
template <class E>
struct Eight {
    E v[8];
    __device__ __forceinline__ void load(const E *p, int left)
    {
        if (left >= 8) {
            __builtin_memcpy(v, p, sizeof(v));
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (E)0.0f;
    }
    __device__ __forceinline__ void store(E *p, int left) const
    {
        if (left >= 8) {
            __builtin_memcpy(p, v, sizeof(v));
            return;
        }
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) p[i] = v[i];
    }
};

template <class E>
__device__ __forceinline__ void store8(void *base, int64_t at, const float (&x)[8], int left)
{
    Eight<E> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = (E)x[i];
    o.store((E *)base + at, left);
}

// Eight weights as fp32, in either type.
template <class H>
__device__ __forceinline__ void load_weight(const void *w, bool w32, int at, int left, float (&out)[8])
{
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = 1.0f;
    } else if (w32) {
        Eight<float> e;
        e.load((const float *)w + at, left);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = e.v[i];
    } else {
        Eight<H> e;
        e.load((const H *)w + at, left);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = (float)e.v[i];
    }
}

// ---------------------------------------------------------------- sums of a row

template <int CTRL>
__device__ __forceinline__ double dpp_d(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)b, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Sum over the aligned group of L lanes that holds this one, in 64 bits, the same in each of them.
template <int L>
__device__ __forceinline__ double lanes_sum(double x)
{
    if (L >= 2) x += dpp_d<kDppQuadXor1>(x);
    if (L >= 4) x += dpp_d<kDppQuadXor2>(x);
    if (L >= 8) x += dpp_d<kDppRowHalfMirror>(x);
    if (L >= 16) x += dpp_d<kDppRowMirror>(x);
    if (L >= 32) x += __shfl_xor(x, 16);
    if (L >= 64) x += __shfl_xor(x, 32);
    return x;
}

template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x)
{
    if (L >= 2) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppQuadXor1, 0xF, 0xF, true));
    if (L >= 4) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppQuadXor2, 0xF, 0xF, true));
    if (L >= 8) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppRowHalfMirror, 0xF, 0xF, true));
    if (L >= 16) x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kDppRowMirror, 0xF, 0xF, true));
    if (L >= 32) x = max(x, (uint32_t)__shfl_xor((int)x, 16));
    if (L >= 64) x = max(x, (uint32_t)__shfl_xor((int)x, 32));
    return x;
}

// The same over a row of L threads, which beyond a wave are the workgroup.  Each call takes its own `lds`
// (one value a wave), so that no barrier stands before it.
template <int L>
__device__ __forceinline__ double row_sum(double x, double *lds)
{
    x = lanes_sum<(L < 64 ? L : 64)>(x);
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = lds[0];
#pragma unroll
        for (int i = 1; i < L / 64; ++i) x += lds[i];
    }
    return x;
}
template <int L>
__device__ __forceinline__ uint32_t row_max(uint32_t x, uint32_t *lds)
{
    x = lanes_max<(L < 64 ? L : 64)>(x);
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
        __syncthreads();
        x = lds[0];
#pragma unroll
        for (int i = 1; i < L / 64; ++i) x = max(x, lds[i]);
    }
    return x;
}

// ---------------------------------------------------------------- dropout's numbers

// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011).  An element's
// number depends on its row and column alone, so the backward pass makes it again and no mask is stored.
struct Philox {
    uint32_t k0, k1, o0, o1;
    __device__ __forceinline__ void init(const DropArgs &d)
    {
        const uint64_t seed = (uint64_t)d.rng[0], o = (uint64_t)d.rng[1] + (uint64_t)d.call;
        k0 = (uint32_t)seed;
        k1 = (uint32_t)(seed >> 32);
        o0 = (uint32_t)o;
        o1 = (uint32_t)(o >> 32);
    }
    __device__ __forceinline__ void four(uint32_t quad, uint32_t row, uint32_t *out) const
    {
        uint32_t a = quad, b = row, c = o0, d = o1, x = k0, y = k1;
#pragma unroll
        for (int i = 0; i < 10; ++i) {
            const uint64_t p = (uint64_t)a * 0xD2511F53u, q = (uint64_t)c * 0xCD9E8D57u;
            a = (uint32_t)(q >> 32) ^ b ^ x;
            c = (uint32_t)(p >> 32) ^ d ^ y;
            b = (uint32_t)q;
            d = (uint32_t)p;
            x += 0x9E3779B9u;
            y += 0xBB67AE85u;
        }
        out[0] = a;
        out[1] = b;
        out[2] = c;
        out[3] = d;
    }
    // of the eight columns from `col` on, a multiple of eight
    __device__ __forceinline__ void eight(int col, int64_t row, uint32_t (&out)[8]) const
    {
        four((uint32_t)col >> 2, (uint32_t)row, out);
        four(((uint32_t)col >> 2) + 1, (uint32_t)row, out + 4);
    }
};

// ---------------------------------------------------------------- 8-bit codes

__device__ __forceinline__ uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The scale of 8-bit integers whose largest magnitude has these bits: top / 127, at least 2^-126 (so that its inverse
// is finite); NaN for an infinity or a NaN.
__device__ __forceinline__ float int8_scale(uint32_t top)
{
    if (top >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    return fmaxf(__uint_as_float(top) / 127.0f, __uint_as_float(0x00800000u));
}

// Four codes: x times the scale's inverse, rounded once to the nearest whole number, ties to even, by the sum with
// 1.5 * 2^23, whose lowest bits then hold it.
__device__ __forceinline__ uint32_t int8_codes4(const float *x, float inverse)
{
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(__builtin_fmaf(x[i], inverse, 12582912.0f));
    return (b[0] & 0xFF) | (b[1] & 0xFF) << 8 | (b[2] & 0xFF) << 16 | b[3] << 24;
}

__device__ __forceinline__ void store_int8(uint8_t *codes, const float (&x)[8], float inverse, bool bad)
{
    uint2 q = make_uint2(int8_codes4(x, inverse), int8_codes4(x + 4, inverse));
    if (bad) q = make_uint2(0, 0);
    *(uint2 *)codes = q;
}

#endif  // __HIPCC__

}  // namespace rgnn
