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

// How rows are made of vectors of eight: of whole ones, ending inside one, or of fewer than eight columns.  Kernels are
// compiled for one of them: with the columns' loads in a branch beside the vectors', loads of one row wait for
// each other (100 000 x 333 fp16, backward: 95 us, apart 75).
enum Fit : int { kWhole, kEnds, kTiny };
inline Fit fit_of(int cols) { return cols % 8 == 0 ? kWhole : cols < 8 ? kTiny : kEnds; }

// The compiler takes these values as new: it keeps them and nothing that it made of them before.
template <class T, int N>
__device__ __forceinline__ void opaque(T (&x)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}

// Eight values of a row from column c on, those behind its `cols` columns zero, from any address of an element: a
// vector load takes any address, at full speed where it is a multiple of its size.  load() only asks for them,
// so that many loads are under way together; settle() comes before their use.  A vector that
// the row does not fill is read as the row's last eight and moved down.
template <class E, Fit FIT>
struct Eight {
    static constexpr int words = sizeof(E) * 2;
    uint32_t raw[words];
    __device__ __forceinline__ void load(const E *row, int c, int cols)
    {
        if constexpr (FIT == kTiny) {
            E e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = row[min(i, cols - 1)];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = c + i < cols ? e[i] : (E)0.0f;
            __builtin_memcpy(raw, e, sizeof(raw));
        } else {
            __builtin_memcpy(raw, row + min(c, cols - 8), sizeof(raw));
        }
    }
    __device__ __forceinline__ void settle(int c, int cols)
    {
        if constexpr (FIT == kTiny) return;
        if constexpr (FIT == kWhole) {
#pragma unroll
            for (int i = 0; i < words; ++i) raw[i] = c < cols ? raw[i] : 0;
            return;
        }
        if (c + 8 <= cols) return;
        const int by = 8 - (cols & 7);            // the same for all lanes whose vector the row ends in: c is whole vectors
        if constexpr (sizeof(E) == 2) {
            if (by & 2)
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[i] = i < 3 ? raw[i + 1] : 0;
            if (by & 4)
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[i] = i < 2 ? raw[i + 2] : 0;
            if (by & 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) raw[i] = raw[i] >> 16 | (i < 3 ? raw[i + 1] << 16 : 0);
        } else {
#pragma unroll
            for (int step = 1; step < 8; step *= 2)
                if (by & step)
#pragma unroll
                    for (int i = 0; i < 8; ++i) raw[i] = i + step < 8 ? raw[i + step] : 0;
        }
#pragma unroll
        for (int i = 0; i < words; ++i) raw[i] = c < cols ? raw[i] : 0;
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(E) == 4) return __uint_as_float(raw[i]);
        else if constexpr (std::is_same<E, __bf16>::value) return __uint_as_float(i & 1 ? raw[i >> 1] & 0xFFFF0000u : raw[i >> 1] << 16);
        else return (float)__builtin_bit_cast(_Float16, (uint16_t)(raw[i >> 1] >> (i & 1) * 16));
    }
};

// Eight results to a row from column c on, those that it has: the last ones in pieces of four, two and one, by whole
// words (selected as elements, they would go through memory).
template <class E, Fit FIT>
__device__ __forceinline__ void store8(void *base, int64_t row, const float (&x)[8], int c, int cols)
{
    typedef E vec __attribute__((ext_vector_type(8)));
    vec v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (E)x[i];
    E *p = (E *)base + row + c;
    const int left = cols & 7;                    // of the vector that the row ends in
    if (c + 8 <= cols) {
        __builtin_memcpy(p, &v, sizeof(v));
    } else if (FIT != kWhole && c < cols) {
        if constexpr (sizeof(E) == 2) {
            i32x4 w = __builtin_bit_cast(i32x4, v);
            if (left & 4) {
                const int2 q = make_int2(w[0], w[1]);
                __builtin_memcpy(p, &q, 8);
                p += 4;
            }
            const int w0 = left & 4 ? w[2] : w[0], w1 = left & 4 ? w[3] : w[1];
            if (left & 2) {
                __builtin_memcpy(p, &w0, 4);
                p += 2;
            }
            const uint16_t last = (uint16_t)(left & 2 ? w1 : w0);
            if (left & 1) __builtin_memcpy(p, &last, 2);
        } else {
            i32x8 w = __builtin_bit_cast(i32x8, v);
            if (left & 4) {
                const i32x4 q = {w[0], w[1], w[2], w[3]};
                __builtin_memcpy(p, &q, 16);
                p += 4;
            }
            const int w0 = left & 4 ? w[4] : w[0], w1 = left & 4 ? w[5] : w[1], w2 = left & 4 ? w[6] : w[2];
            if (left & 2) {
                const int2 q = make_int2(w0, w1);
                __builtin_memcpy(p, &q, 8);
                p += 2;
            }
            const int last = left & 2 ? w2 : w0;
            if (left & 1) __builtin_memcpy(p, &last, 4);
        }
    }
}

// Eight weights as fp32, in either type.
template <class H, Fit FIT>
__device__ __forceinline__ void load_weight(const void *w, bool w32, int c, int cols, float (&out)[8])
{
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = 1.0f;
    } else if (w32) {
        Eight<float, FIT> e;
        e.load((const float *)w, c, cols);
        e.settle(c, cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = e.at(i);
    } else {
        Eight<H, FIT> e;
        e.load((const H *)w, c, cols);
        e.settle(c, cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = e.at(i);
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
            a = (uint32_t)__builtin_amdgcn_bitop3_b32((int)(q >> 32), (int)b, (int)x, 0x96);      // exclusive or of three
            c = (uint32_t)__builtin_amdgcn_bitop3_b32((int)(p >> 32), (int)d, (int)y, 0x96);
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

__device__ __forceinline__ void store_e4m3(uint8_t *codes, const float (&x)[8], int byte)
{
    const float inv = e4m3_scale_inverse(byte);
    uint2 q = make_uint2(e4m3_codes4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), e4m3_codes4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    if (byte == 255) q = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
    *(uint2 *)codes = q;
}

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
