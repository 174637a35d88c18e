// int8_quantize.hip -- rows and weights as 8-bit integers, with a scale for each row (token) and for each
// output of a type's weight (channel): scale = max |x| / 127, code = round(x (1 / scale)).
//
// A row stays in registers between its maximum and its codes.  A weight's columns are read twice, for
// their maxima and for the codes, which turn over in LDS to rows of k.
#include <algorithm>

#include "rows.h"

namespace rgnn {

namespace {

template <class E, bool WHOLE, int L, int NV>
__global__ __launch_bounds__(L > 256 ? L : 256) void int8_rows_kernel(const E *X, int64_t rows, int64_t ldx, int K, uint8_t *codes,
                                                                      float *scales)
{
    constexpr int PER = L >= 256 ? 1 : 256 / L;
    __shared__ uint32_t tops[L > 64 ? L / 64 : 1];
    const int64_t row = flat_block() * (int64_t)PER + (PER > 1 ? threadIdx.x / L : 0);
    if (row >= rows) return;
    const int lane = threadIdx.x % L, kp = fp8_width(K);
    Eight<E, WHOLE> x[NV];
    uint32_t top = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) x[v].load(X + row * ldx, (v * L + lane) * 8, K);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        x[v].settle((v * L + lane) * 8, K);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(x[v].at(i)));
    }
    const float scale = int8_scale(row_max<L>(top, tops)), inverse = 1.0f / scale;
    if (lane == 0) scales[row] = scale;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * L + lane) * 8;
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = x[v].at(i);
        if (c < kp) store_int8(codes + row * kp + c, f, inverse, scale != scale);
    }
}

// Rows that registers do not hold are read twice.
template <class E>
__global__ __launch_bounds__(1024) void int8_long_rows_kernel(const E *X, int64_t rows, int64_t ldx, int K, uint8_t *codes, float *scales)
{
    __shared__ uint32_t tops[16];
    const int64_t row = flat_block();
    if (row >= rows) return;
    const int kp = fp8_width(K);
    uint32_t top = 0;
    for (int c = threadIdx.x * 8; c < K; c += 8192) {
        Eight<E, false> x;
        x.load(X + row * ldx, c, K);
        x.settle(c, K);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(x.at(i)));
    }
    const float scale = int8_scale(row_max<1024>(top, tops)), inverse = 1.0f / scale;
    if (threadIdx.x == 0) scales[row] = scale;
    for (int c = threadIdx.x * 8; c < kp; c += 8192) {
        Eight<E, false> x;
        float f[8];
        x.load(X + row * ldx, c, K);
        x.settle(c, K);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = x.at(i);
        store_int8(codes + row * kp + c, f, inverse, scale != scale);
    }
}

// A workgroup takes 64 outputs of one type: eight threads across, 32 rows of k at a time for the maxima, then 128 for
// the codes.
template <class E, bool WHOLE>
__global__ __launch_bounds__(256) void int8_weights_kernel(const E *W, int K, int N, int kp, uint8_t *codes, float *scales)
{
    __shared__ __attribute__((aligned(16))) uint8_t turn[64 * 144];
    __shared__ uint32_t tops[32][64];
    __shared__ float inverse[64];
    const int tid = threadIdx.x, across = (tid & 7) * 8, down = tid >> 3;
    const int64_t t = blockIdx.y;
    const int n0 = blockIdx.x * 64, n = n0 + across;
    const E *w = W + t * K * N;
    uint32_t top[8] = {};
#pragma unroll 4
    for (int k = down; k < K; k += 32) {
        Eight<E, WHOLE> x;
        x.load(w + (int64_t)k * N, n, N);
        x.settle(n, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) top[i] = max(top[i], magnitude_bits(x.at(i)));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) tops[down][across + i] = top[i];
    __syncthreads();
    if (tid < 64) {
        uint32_t m = 0;
        for (int i = 0; i < 32; ++i) m = max(m, tops[i][tid]);
        const float scale = int8_scale(m);
        inverse[tid] = scale != scale ? 0.0f : 1.0f / scale;      // 0: codes of 0
        if (n0 + tid < N) scales[t * N + n0 + tid] = scale;
    }
    __syncthreads();
    float inv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) inv[i] = inverse[across + i];
    for (int k0 = 0; k0 < kp; k0 += 128) {
        Eight<E, WHOLE> x[4];                    // four k side by side
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q].load(w + (int64_t)min(k0 + down * 4 + q, K - 1) * N, n, N);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q].settle(n, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) b[q] = inv[i] == 0.0f || k0 + down * 4 + q >= K ? 0 : __float_as_uint(__builtin_fmaf(x[q].at(i), inv[i], 12582912.0f));
            *(uint32_t *)(turn + (across + i) * 144 + down * 4) = (b[0] & 0xFF) | (b[1] & 0xFF) << 8 | (b[2] & 0xFF) << 16 | b[3] << 24;
        }
        __syncthreads();
#pragma unroll
        for (int c = tid; c < 64 * 8; c += 256)
            if (n0 + (c >> 3) < N)
                *(i32x4 *)(codes + (t * N + n0 + (c >> 3)) * kp + k0 + (c & 7) * 16) = *(const i32x4 *)(turn + (c >> 3) * 144 + (c & 7) * 16);
        __syncthreads();
    }
}

template <class E, int L, int NV>
void launch_shape(const E *X, int64_t rows, int64_t ldx, int K, uint8_t *codes, float *scales, hipStream_t s)
{
    constexpr int PER = L >= 256 ? 1 : 256 / L;
    const dim3 g = flat_grid((rows + PER - 1) / PER), b(L > 256 ? L : 256);
    if (whole_vectors(K)) hipLaunchKernelGGL((int8_rows_kernel<E, true, L, NV>), g, b, 0, s, X, rows, ldx, K, codes, scales);
    else hipLaunchKernelGGL((int8_rows_kernel<E, false, L, NV>), g, b, 0, s, X, rows, ldx, K, codes, scales);
}

template <class E>
void rows_of(const void *p, int64_t rows, int64_t ldx, int K, void *c, float *scales, hipStream_t s)
{
    const E *X = (const E *)p;
    uint8_t *codes = (uint8_t *)c;
    if (K <= 128) launch_shape<E, 16, 1>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 256) launch_shape<E, 32, 1>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 512) launch_shape<E, 64, 1>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 1024) launch_shape<E, 64, 2>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 2048) launch_shape<E, 256, 1>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 4096) launch_shape<E, 256, 2>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 8192) launch_shape<E, 256, 4>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 16384) launch_shape<E, 1024, 2>(X, rows, ldx, K, codes, scales, s);
    else hipLaunchKernelGGL((int8_long_rows_kernel<E>), flat_grid(rows), dim3(1024), 0, s, X, rows, ldx, K, codes, scales);
}

template <class E>
void weights_of(const void *W, int T, int K, int N, void *codes, float *scales, hipStream_t s)
{
    const dim3 g((uint32_t)((N + 63) / 64), (uint32_t)T);
    if (whole_vectors(N)) hipLaunchKernelGGL((int8_weights_kernel<E, true>), g, dim3(256), 0, s, (const E *)W, K, N, fp8_width(K), (uint8_t *)codes, scales);
    else hipLaunchKernelGGL((int8_weights_kernel<E, false>), g, dim3(256), 0, s, (const E *)W, K, N, fp8_width(K), (uint8_t *)codes, scales);
}

}  // namespace

rgnn_status launch_int8_rows(int dtype, const void *X, int64_t rows, int64_t ldx, int K, void *codes, float *scales, hipStream_t s)
{
    {
        LaunchScope ls("int8_rows", s);
        if (dtype == RGNN_F32) rows_of<float>(X, rows, ldx, K, codes, scales, s);
        else if (dtype == RGNN_BF16) rows_of<__bf16>(X, rows, ldx, K, codes, scales, s);
        else rows_of<_Float16>(X, rows, ldx, K, codes, scales, s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "int8_rows launch");
}

rgnn_status launch_int8_weights(int dtype, const void *W, int T, int K, int N, void *codes, float *scales, hipStream_t s)
{
    {
        LaunchScope ls("int8_weights", s);
        if (dtype == RGNN_F32) weights_of<float>(W, T, K, N, codes, scales, s);
        else if (dtype == RGNN_BF16) weights_of<__bf16>(W, T, K, N, codes, scales, s);
        else weights_of<_Float16>(W, T, K, N, codes, scales, s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "int8_weights launch");
}

}  // namespace rgnn
