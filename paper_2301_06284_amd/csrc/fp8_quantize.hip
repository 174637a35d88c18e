// fp8_quantize.hip -- rows and weights in 8 bits (e4m3) with a power-of-two scale for
// each block of 128.
//
// With a power of two for the scale s, x / s is exact, so a code is one rounding of x
// and the result does not depend on how a quotient is rounded; the matrix cores take the
// scale's exponent byte as an operand.  The least s with max |x| <= 448 s comes from the
// bits of the largest magnitude: 448 = 1.75 * 2^8, so the exponent goes up where the
// mantissa lies above 1.75 (0x600000), which adding 0x1FFFFF carries into it.  The maximum
// is taken over bits as integers, where a NaN or an infinity is larger than any number.
//
// Bound by memory: every element is read once and a byte written.  Measured, bf16: rows 8192 x 4096 19
// us (5.2 TB/s), weights 16 x 2048 x 1536 29 us (5.2 TB/s), 8 rows of 2048 2.8 us (a launch).
#include <algorithm>

#include "linear_ops.h"

namespace rgnn {

namespace {

// scale byte of a block whose largest magnitude has these bits
__device__ __forceinline__ int scale_byte(uint32_t top)
{
    if (top >= 0x7F800000u) return 255;
    const int e = (int)((top + 0x1FFFFFu) >> 23) - 8;
    return e < 1 ? 1 : e;
}
// 1 / scale, exact; NaN for byte 255
__device__ __forceinline__ float scale_inverse(int byte)
{
    return byte == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float((uint32_t)(254 - byte) << 23);
}

// four codes of four values (|x| <= 448, or NaN)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// Eight values of a row from column k on, zero behind K.
template <class E, bool VEC>
__device__ __forceinline__ void load8(const E *row, int64_t k, int K, float x[8])
{
    if (VEC && k + 8 <= K) {
        E v[8];
        *(i32x4 *)v = *(const i32x4 *)(row + k);
        if constexpr (sizeof(E) == 4) *(i32x4 *)(v + 4) = *(const i32x4 *)(row + k + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = k + i < K ? (float)row[k + i] : 0.0f;
}

// A wave takes 512 elements of a row: 8 a lane, 16 lanes a block, four blocks, which is one
// word of scales.
template <class E, bool VEC>
__global__ __launch_bounds__(256) void fp8_rows_kernel(const E *X, int64_t rows, int64_t ldx, int K, int Kp, int words,
                                                       uint8_t *codes, uint8_t *scales)
{
    const int lane = threadIdx.x & 63;
    const int64_t task = flat_block() * (int64_t)4 + (threadIdx.x >> 6);
    if (task >= rows * words) return;
    const int64_t row = task / words;
    const int w = (int)(task % words);
    const int64_t k = (int64_t)w * 512 + lane * 8;
    float x[8];
    load8<E, VEC>(X + row * ldx, k, K, x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, magnitude(x[i]));
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const int byte = k < Kp ? scale_byte(top) : 127;
    if (k < Kp) {
        const float inv = scale_inverse(byte);
        uint2 q;
        q.x = codes4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
        q.y = codes4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
        if (byte == 255) q = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
        *(uint2 *)(codes + row * Kp + k) = q;
    }
    if ((lane & 15) == 0) scales[(row * words + w) * 4 + (lane >> 4)] = (uint8_t)byte;
}

// A workgroup takes one 128 x 128 block of a weight: a thread 8 k x 8 n, so that it
// holds whole pieces of k for each n; the codes turn over in LDS to rows of 128 k.
template <class E, bool VEC>
__global__ __launch_bounds__(256) void fp8_weights_kernel(const E *W, int K, int N, int Kp, int words, int nb,
                                                          uint8_t *codes, uint8_t *scales)
{
    __shared__ __attribute__((aligned(16))) uint8_t turn[128 * 144];
    __shared__ uint32_t tops[4];
    const int tid = threadIdx.x, kb = blockIdx.x, jb = blockIdx.y;
    const int64_t t = blockIdx.z;
    uint8_t *sc = scales + ((t * nb + jb) * words) * 4;
    if (kb * 128 >= Kp) {                 // behind the last block
        if (tid == 0) sc[kb] = 127;
        return;
    }
    const int n0 = jb * 128 + (tid & 15) * 8, k0 = kb * 128 + (tid >> 4) * 8;
    float x[8][8];                        // [k][n]
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (k0 + i < K) load8<E, VEC>(W + (t * K + k0 + i) * N, n0, N, x[i]);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(x[i][j]));
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    __syncthreads();
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    const int byte = scale_byte(top);
    const float inv = scale_inverse(byte);
    if (tid == 0) sc[kb] = (uint8_t)byte;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint2 q;
        q.x = codes4(x[0][j] * inv, x[1][j] * inv, x[2][j] * inv, x[3][j] * inv);
        q.y = codes4(x[4][j] * inv, x[5][j] * inv, x[6][j] * inv, x[7][j] * inv);
        if (byte == 255) q = make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu);
        *(uint2 *)(turn + ((tid & 15) * 8 + j) * 144 + (tid >> 4) * 8) = q;
    }
    __syncthreads();
    for (int c = tid; c < 128 * 8; c += 256) {
        const int n = jb * 128 + (c >> 3);
        if (n < N) *(i32x4 *)(codes + (t * N + n) * Kp + kb * 128 + (c & 7) * 16) = *(const i32x4 *)(turn + (c >> 3) * 144 + (c & 7) * 16);
    }
}

template <class E>
void rows_of(const void *X, int64_t rows, int64_t ldx, int K, int Kp, int words, uint8_t *c, uint8_t *sc, hipStream_t s)
{
    const bool vec = ((uintptr_t)X % 16 == 0) && (ldx * sizeof(E)) % 16 == 0;
    const dim3 g = flat_grid((rows * words + 3) / 4);
    if (vec) hipLaunchKernelGGL((fp8_rows_kernel<E, true>), g, dim3(256), 0, s, (const E *)X, rows, ldx, K, Kp, words, c, sc);
    else hipLaunchKernelGGL((fp8_rows_kernel<E, false>), g, dim3(256), 0, s, (const E *)X, rows, ldx, K, Kp, words, c, sc);
}

template <class E>
void weights_of(const void *W, int T, int K, int N, int Kp, int words, uint8_t *c, uint8_t *sc, hipStream_t s)
{
    const bool vec = ((uintptr_t)W % 16 == 0) && ((int64_t)N * sizeof(E)) % 16 == 0;
    const int nb = (N + 127) / 128;
    const dim3 g((uint32_t)words * 4, (uint32_t)nb, (uint32_t)T);
    if (vec) hipLaunchKernelGGL((fp8_weights_kernel<E, true>), g, dim3(256), 0, s, (const E *)W, K, N, Kp, words, nb, c, sc);
    else hipLaunchKernelGGL((fp8_weights_kernel<E, false>), g, dim3(256), 0, s, (const E *)W, K, N, Kp, words, nb, c, sc);
}

}  // namespace

rgnn_status launch_fp8_rows(int dtype, const void *X, int64_t rows, int64_t ldx, int K, void *codes, uint8_t *scales, hipStream_t s)
{
    const int Kp = fp8_width(K), words = fp8_scales(K) / 4;
    if ((rows * words + 3) / 4 >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many rows");
    {
        LaunchScope ls("fp8_rows", s);
        if (dtype == RGNN_F32) rows_of<float>(X, rows, ldx, K, Kp, words, (uint8_t *)codes, scales, s);
        else if (dtype == RGNN_BF16) rows_of<__bf16>(X, rows, ldx, K, Kp, words, (uint8_t *)codes, scales, s);
        else rows_of<_Float16>(X, rows, ldx, K, Kp, words, (uint8_t *)codes, scales, s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "fp8_rows launch");
}

rgnn_status launch_fp8_weights(int dtype, const void *W, int T, int K, int N, void *codes, uint8_t *scales, hipStream_t s)
{
    const int Kp = fp8_width(K), words = fp8_scales(K) / 4;
    if ((N + 127) / 128 > 65535) return fail(RGNN_ERANGE, "weights too wide");
    {
        LaunchScope ls("fp8_weights", s);
        if (dtype == RGNN_F32) weights_of<float>(W, T, K, N, Kp, words, (uint8_t *)codes, scales, s);
        else if (dtype == RGNN_BF16) weights_of<__bf16>(W, T, K, N, Kp, words, (uint8_t *)codes, scales, s);
        else weights_of<_Float16>(W, T, K, N, Kp, words, (uint8_t *)codes, scales, s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "fp8_weights launch");
}

}  // namespace rgnn
