// int8_quantize.hip -- rows and weights as 8-bit integers, with a scale for each row (token) and for each
// output of a type's weight (channel): scale = max |x| / 127, code = round(x (1 / scale)).
//
// A row stays in registers between its maximum and its codes, and so do a weight's columns up to 4096 k in 16 bits (2048 in
// fp32; of the longest, 16-bit outputs that end inside a vector spill three registers); longer ones are read twice.  The weights' codes turn over in LDS to rows of k.
//
// Bound by memory.  Measured, bf16: rows 8192 x 4096 17 us (5.8 TB/s), 8 rows of 2048 2.6; weights 16 x 2048 x 1536
// 39 us (3.8 TB/s: every workgroup loads first and stores last), 4096 x 4096 18, 4 x 5000 x 3000 (read twice) 74.
#include <algorithm>

#include "rows.h"

namespace rgnn {

namespace {

template <class E, Fit FIT, int L, int NV>
__global__ __launch_bounds__(L > 64 ? L : 256) void int8_rows_kernel(const E *X, int64_t rows, int64_t ldx, int K, uint8_t *codes,
                                                                      float *scales)
{
    constexpr int PER = L > 64 ? 1 : 256 / L;
    __shared__ uint32_t tops[L > 64 ? L / 64 : 1];
    const int64_t row = flat_block() * (int64_t)PER + (PER > 1 ? threadIdx.x / L : 0);
    if (row >= rows) return;
    const int lane = threadIdx.x % L, kp = fp8_width(K);
    Eight<E, FIT> x[NV];
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
        Eight<E, kEnds> x;
        x.load(X + row * ldx, c, K);
        x.settle(c, K);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(x.at(i)));
    }
    const float scale = int8_scale(row_max<1024>(top, tops)), inverse = 1.0f / scale;
    if (threadIdx.x == 0) scales[row] = scale;
    for (int c = threadIdx.x * 8; c < kp; c += 8192) {
        Eight<E, kEnds> x;
        float f[8];
        x.load(X + row * ldx, c, K);
        x.settle(c, K);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = x.at(i);
        store_int8(codes + row * kp + c, f, inverse, scale != scale);
    }
}

// The largest magnitudes of eight columns so far, 16-bit ones two a word: bits of magnitudes order like whole numbers.
template <class E>
struct Tops {
    static constexpr int words = Eight<E, kWhole>::words;
    typedef uint16_t pair __attribute__((ext_vector_type(2)));
    uint32_t raw[words];
    __device__ __forceinline__ void see(const uint32_t (&x)[words])
    {
#pragma unroll
        for (int i = 0; i < words; ++i) {
            if constexpr (sizeof(E) == 4) raw[i] = max(raw[i], x[i] & 0x7FFFFFFFu);
            else raw[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(pair, raw[i]), __builtin_bit_cast(pair, x[i] & 0x7FFF7FFFu)));
        }
    }
    __device__ __forceinline__ uint32_t bits(int i) const      // as fp32
    {
        if constexpr (sizeof(E) == 4) return raw[i];
        else return __float_as_uint(((const Eight<E, kWhole> &)raw).at(i));
    }
};

// A workgroup takes 32 outputs of one type with all their k, which stay in registers, as they came, from the maxima to
// the codes: four threads across, P times four k a thread.  Loads have one base for all lanes and 32-bit offsets that the
// P passes share (`k_bytes`: from one k to the next; KS of them stay below 2^32), and no more registers than let a second
// workgroup of the CU load while this one computes.
template <class E, Fit FIT, int TH, int P>
__global__ __launch_bounds__(TH, sizeof(E) == 4 ? 2 : 4) void int8_weights_kernel(const char *W, int T, int K, int N, int kp, uint32_t k_bytes, uint8_t *codes,
                                                                                  float *scales)
{
    constexpr int KS = TH, ROW = KS + 16;            // k of one pass; bytes of an output's codes in LDS
    __shared__ __attribute__((aligned(16))) uint8_t turn[32 * ROW];
    __shared__ uint32_t tops[TH / 64][32];
    __shared__ float inverse[32];
    const int tid = threadIdx.x, across = (tid & 3) * 8, down = (tid >> 2) * 4;
    // Sixteen workgroups are eight pairs, the two of a pair on one XCD: its L2 fetches lines of 128 bytes, which are two
    // workgroups' columns.
    const uint32_t pairs = (uint32_t)(N + 63) / 64, pair = blockIdx.x / 16 * 8 + (blockIdx.x & 7), t = pair / pairs;
    const int n0 = (int)(pair - t * pairs) * 64 + (blockIdx.x >> 3 & 1) * 32, n = n0 + across;
    if (t >= (uint32_t)T || n0 >= N) return;
    const char *w = W + t * K * (int64_t)k_bytes;
    const uint32_t at = (uint32_t)min(n, N - 8) * (uint32_t)sizeof(E);
    Eight<E, FIT> x[P][4];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int first = min(p * KS, (K - 1) / 4 * 4), rows = K - first;      // behind K the last one again: no new maximum
        const char *base = w + (int64_t)first * k_bytes;
#pragma unroll
        for (int q = 0; q < 4; ++q) __builtin_memcpy(x[p][q].raw, base + (at + (uint32_t)min(down + q, rows - 1) * k_bytes), sizeof(x[p][q].raw));
    }
    Tops<E> top = {};
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (FIT != kWhole) x[p][q].settle(n, N);
            top.see(x[p][q].raw);
            opaque(x[p][q].raw);
        }
#pragma unroll
    for (int d = 4; d < 64; d <<= 1) {
        uint32_t other[Tops<E>::words];
#pragma unroll
        for (int i = 0; i < Tops<E>::words; ++i) other[i] = (uint32_t)__shfl_xor((int)top.raw[i], d);
        top.see(other);
    }
    if ((tid & 63) < 4)
#pragma unroll
        for (int i = 0; i < 8; ++i) tops[tid >> 6][across + i] = top.bits(i);
    __syncthreads();
    if (tid < 32) {
        uint32_t m = 0;
        for (int i = 0; i < TH / 64; ++i) m = max(m, tops[i][tid]);
        const float scale = int8_scale(m);
        inverse[tid] = scale != scale ? 0.0f : 1.0f / scale;      // 0: codes of 0
        if (n0 + tid < N) scales[(int64_t)t * N + n0 + tid] = scale;
    }
    __syncthreads();
    float inv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) inv[i] = inverse[across + i];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int k0 = p * KS;
        if (k0 >= kp) break;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                b[q] = inv[i] == 0.0f || k0 + down + q >= K ? 0 : __float_as_uint(__builtin_fmaf(x[p][q].at(i), inv[i], 12582912.0f));
            *(uint32_t *)(turn + (across + i) * ROW + down) = (b[0] & 0xFF) | (b[1] & 0xFF) << 8 | (b[2] & 0xFF) << 16 | b[3] << 24;
        }
        __syncthreads();
#pragma unroll
        for (int c = tid; c < 32 * KS / 16; c += TH) {
            const int row = c / (KS / 16), to = c % (KS / 16) * 16;
            if (n0 + row < N && k0 + to < kp) *(i32x4 *)(codes + ((int64_t)t * N + n0 + row) * kp + k0 + to) = *(const i32x4 *)(turn + row * ROW + to);
        }
        if (p + 1 < P) __syncthreads();
    }
}

// Longer k are read twice.  A workgroup takes 64 outputs of one type: eight threads across, TH / 8 rows of k at a time for the maxima, then
// four times as many for the codes, which turn over in LDS.  The second reading comes from L2 or the last-level cache.
template <class E, Fit FIT, int TH>
__global__ __launch_bounds__(TH) void int8_long_weights_kernel(const E *W, int K, int N, int kp, uint8_t *codes, float *scales)
{
    constexpr int DOWN = TH / 8, KS = DOWN * 4, ROW = KS + 16;      // k of a turn; bytes of an output's codes in LDS
    __shared__ __attribute__((aligned(16))) uint8_t turn[64 * ROW];
    __shared__ uint32_t tops[TH / 64][64];
    __shared__ float inverse[64];
    const int tid = threadIdx.x, across = (tid & 7) * 8, down = tid >> 3;
    const int64_t t = blockIdx.y;
    const int n0 = blockIdx.x * 64, n = n0 + across;
    const E *w = W + t * K * N;
    uint32_t top[8] = {};
#pragma unroll 4
    for (int k = down; k < K; k += DOWN) {
        Eight<E, FIT> x;
        x.load(w + (int64_t)k * N, n, N);
        x.settle(n, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) top[i] = max(top[i], magnitude_bits(x.at(i)));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int d = 8; d < 64; d <<= 1) top[i] = max(top[i], (uint32_t)__shfl_xor((int)top[i], d));
        if ((tid & 63) < 8) tops[tid >> 6][across + i] = top[i];
    }
    __syncthreads();
    if (tid < 64) {
        uint32_t m = 0;
        for (int i = 0; i < TH / 64; ++i) m = max(m, tops[i][tid]);
        const float scale = int8_scale(m);
        inverse[tid] = scale != scale ? 0.0f : 1.0f / scale;      // 0: codes of 0
        if (n0 + tid < N) scales[t * N + n0 + tid] = scale;
    }
    __syncthreads();
    float inv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) inv[i] = inverse[across + i];
    for (int k0 = 0; k0 < kp; k0 += KS) {
        const int first = k0 + down * 4;
        Eight<E, FIT> x[4];                    // four k side by side
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q].load(w + (int64_t)min(first + q, K - 1) * N, n, N);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q].settle(n, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) b[q] = inv[i] == 0.0f || first + q >= K ? 0 : __float_as_uint(__builtin_fmaf(x[q].at(i), inv[i], 12582912.0f));
            *(uint32_t *)(turn + (across + i) * ROW + down * 4) = (b[0] & 0xFF) | (b[1] & 0xFF) << 8 | (b[2] & 0xFF) << 16 | b[3] << 24;
        }
        __syncthreads();
#pragma unroll
        for (int c = tid; c < 64 * KS / 16; c += TH) {
            const int row = c / (KS / 16), at = c % (KS / 16) * 16;
            if (n0 + row < N && k0 + at < kp) *(i32x4 *)(codes + (t * N + n0 + row) * kp + k0 + at) = *(const i32x4 *)(turn + row * ROW + at);
        }
        __syncthreads();
    }
}

template <class E, int L, int NV>
void launch_shape(const E *X, int64_t rows, int64_t ldx, int K, uint8_t *codes, float *scales, hipStream_t s)
{
    constexpr int PER = L > 64 ? 1 : 256 / L;
    const dim3 g = flat_grid((rows + PER - 1) / PER), b(L > 64 ? L : 256);
    const Fit fit = fit_of(K);
    if (fit == kWhole) hipLaunchKernelGGL((int8_rows_kernel<E, kWhole, L, NV>), g, b, 0, s, X, rows, ldx, K, codes, scales);
    else if (fit == kEnds) hipLaunchKernelGGL((int8_rows_kernel<E, kEnds, L, NV>), g, b, 0, s, X, rows, ldx, K, codes, scales);
    else if constexpr (L == 16) hipLaunchKernelGGL((int8_rows_kernel<E, kTiny, L, NV>), g, b, 0, s, X, rows, ldx, K, codes, scales);
}

// Two vectors of eight a thread measured fastest, one up to 256 and of 1025 to 2048 columns (bf16: 80 000 x 264 12.9 us, one
// vector of 64 threads 15.5; 8000 x 4096 16.1, 512 threads 18.2; 4000 x 8192 16.1, 1024 threads 18.9).
template <class E>
void rows_of(const void *p, int64_t rows, int64_t ldx, int K, void *c, float *scales, hipStream_t s)
{
    const E *X = (const E *)p;
    uint8_t *codes = (uint8_t *)c;
    if (K <= 128) launch_shape<E, 16, 1>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 256) launch_shape<E, 32, 1>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 512) launch_shape<E, 32, 2>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 1024) launch_shape<E, 64, 2>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 2048) launch_shape<E, 256, 1>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 4096) launch_shape<E, 256, 2>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 8192) launch_shape<E, 512, 2>(X, rows, ldx, K, codes, scales, s);
    else if (K <= 16384) launch_shape<E, 1024, 2>(X, rows, ldx, K, codes, scales, s);
    else hipLaunchKernelGGL((int8_long_rows_kernel<E>), flat_grid(rows), dim3(1024), 0, s, X, rows, ldx, K, codes, scales);
}

template <class E, Fit FIT>
void weights_of(const E *W, int T, int K, int N, uint8_t *codes, float *scales, hipStream_t s)
{
    const int kp = fp8_width(K);
    const uint64_t k_bytes = (uint64_t)N * sizeof(E);
    const int64_t pairs = (int64_t)T * ((N + 63) / 64);
    const dim3 g64((uint32_t)((N + 63) / 64), (uint32_t)T);
    auto once = [&](auto kernel, int th) { hipLaunchKernelGGL(kernel, dim3((uint32_t)((pairs + 7) / 8 * 16)), dim3(th), 0, s, (const char *)W, T, K, N, kp, (uint32_t)k_bytes, codes, scales); };
    if (FIT == kTiny || kp > (sizeof(E) == 2 ? 4096 : 2048) || k_bytes * 1024 >= (uint64_t(1) << 32) || pairs >= (1 << 20)) {
        hipLaunchKernelGGL((int8_long_weights_kernel<E, FIT, 1024>), g64, dim3(1024), 0, s, W, K, N, kp, codes, scales);
    } else if constexpr (FIT != kTiny) {
        if (kp <= 256) once(int8_weights_kernel<E, FIT, 256, 1>, 256);
        else if (kp <= 512) once(int8_weights_kernel<E, FIT, 256, 2>, 256);
        else if (kp <= 1024) once(int8_weights_kernel<E, FIT, 512, 2>, 512);
        else if (kp <= 2048) once(int8_weights_kernel<E, FIT, 512, 4>, 512);
        else if constexpr (sizeof(E) == 2) once(int8_weights_kernel<E, FIT, 1024, 4>, 1024);
    }
}

template <class E>
void weights_any(const void *W, int T, int K, int N, void *codes, float *scales, hipStream_t s)
{
    const Fit fit = fit_of(N);
    if (fit == kWhole) weights_of<E, kWhole>((const E *)W, T, K, N, (uint8_t *)codes, scales, s);
    else if (fit == kEnds) weights_of<E, kEnds>((const E *)W, T, K, N, (uint8_t *)codes, scales, s);
    else weights_of<E, kTiny>((const E *)W, T, K, N, (uint8_t *)codes, scales, s);
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
        if (dtype == RGNN_F32) weights_any<float>(W, T, K, N, codes, scales, s);
        else if (dtype == RGNN_BF16) weights_any<__bf16>(W, T, K, N, codes, scales, s);
        else weights_any<_Float16>(W, T, K, N, codes, scales, s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "int8_weights launch");
}

}  // namespace rgnn
