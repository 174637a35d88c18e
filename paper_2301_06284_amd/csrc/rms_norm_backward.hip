// rms_norm_backward.hip -- gradients of the root-mean-square norm with residual and dropout.
//
// With n = r s and g = dY w: dr = s (g - n mean(g n)) + dsum, the residual's gradient; dX = D'(dr), whose kept
// values the generator tells again; dw = sum over the rows of dY n.  A row is read once and stays in registers, up to 16 384 columns.
// A workgroup takes every G-th group of rows and keeps dw of its columns in registers to the end, then
// writes it to the workspace; a second launch adds the G rows there in 64 bits, in their order, so that results are
// reproducible.
//
// Bound by memory.  Measured, with d_sum, dX and d_residual, both launches: 16 384 x 2048 bf16 with an fp32 sum and dropout 110 us
// (4.9 TB/s), 15 000 x 2048 bf16 58 (5.3), 8000 x 4096 65 (5.0), 100 000 x 333 fp16 77 (4.3), 8 x 2048 6.  One vector a lane takes 70 to
// 105 registers up to 2048 columns (to 116 beyond), which leaves four workgroups of 256 threads or more on a CU; bounds for six spill and
// take 1.4 to 2.5 times as long.  Two vectors a lane (513 to 1024 columns) take 128 to 173, which leaves two to four;
// memory is busy all the same (20 000 x 768 bf16 with an fp32 sum and dropout 45 to 48 us, 5.1 TB/s; 30 000 x 1024 100, 4.9, all bf16
// 55, 5.5; 30 000 x 1001 fp16 63, 4.7).  1024 threads of two vectors (8193 to 16 384 columns) have 128 at most: 16-bit dY and
// sum fit (2000 x 16 000 bf16 75 us, 4.2 TB/s); both fp32, or one of them with dropout, spill up to 52 (fp32 sum and
// dropout 122 us, 4.2; all fp32 145, 4.4, with dropout 169, 3.8, and 16 001 columns 183, 3.5).
#include <algorithm>

#include "rows.h"

namespace rgnn {

namespace {

constexpr int kLong = 32768;         // columns whose dw LDS holds

// Rows of a workgroup: several short ones, of 1 to 64 lanes each.
int rows_of_group(int cols) { return cols <= 8 ? 256 : cols <= 32 ? 64 : cols <= 64 ? 32 : cols <= 128 ? 16 : cols <= 256 ? 8 : cols <= 1024 ? 4 : 1; }
// As many workgroups as the CUs hold at a time: 1024 are four on each (1280, or fewer of them with equal turns,
// 3 to 8 % slower).  At 513 to 1024 columns the registers let 512 or more of the 1024 run at a time, and the others follow.
int64_t groups_of(int64_t rows, int cols)
{
    const int per = rows_of_group(cols);
    return std::min<int64_t>((rows + per - 1) / per, cols <= 2048 ? 1024 : cols <= 4096 ? 512 : 256);
}

template <class H, Fit FIT>
__device__ __forceinline__ void store_typed(void *base, bool f32, int64_t row, const float (&x)[8], int c, int cols)
{
    if (f32) store8<float, FIT>(base, row, x, c, cols);
    else store8<H, FIT>(base, row, x, c, cols);
}

// dX of eight columns from dr, and both stored.
template <class H, class RT, Fit FIT, bool DROP>
__device__ __forceinline__ void store_gradients(const NormBackwardArgs &a, const Philox &gen, int64_t row, int c, float (&dr)[8])
{
    if (a.dres) store8<RT, FIT>(a.dres, row * a.lddr, dr, c, a.cols);
    if (!a.dX) return;
    if constexpr (DROP) {
        uint32_t word[8];
        gen.eight(c, row, word);
#pragma unroll
        for (int i = 0; i < 8; ++i) dr[i] = word[i] > a.drop.below ? dr[i] * a.drop.factor : 0.0f;
    }
    store_typed<H, FIT>(a.dX, a.dx32, row * a.lddx, dr, c, a.cols);
}

template <class H, bool DY32, bool R32, Fit FIT, bool DROP, int L, int NV>
__global__ __launch_bounds__(L > 256 ? L : 256) void rms_norm_backward_kernel(NormBackwardArgs a)
{
#pragma clang fp contract(off)
    typedef typename std::conditional<DY32, float, H>::type YT;
    typedef typename std::conditional<R32, float, H>::type RT;
    constexpr int PER = L >= 256 ? 1 : 256 / L;
    __shared__ double sums[2][L > 64 ? L / 64 : 1];
    __shared__ float part[PER > 1 ? 4 * L * NV * 8 : 1];
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    Philox gen;
    if (DROP) gen.init(a.drop);
    float w[NV][8], dw[NV][8] = {};
#pragma unroll
    for (int v = 0; v < NV; ++v) load_weight<H, FIT>(a.w, a.w32, (v * L + lane) * 8, a.cols, w[v]);
    int turn = 0;
    for (int64_t row = blockIdx.x * (int64_t)PER + group; row < a.rows; row += gridDim.x * (int64_t)PER, turn ^= 1) {
        Eight<YT, FIT> dy[NV];
        Eight<RT, FIT> r[NV], ds[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * L + lane) * 8;
            dy[v].load((const YT *)a.dY + row * a.lddy, c, a.cols);
            r[v].load((const RT *)a.r + row * a.ldr, c, a.cols);
        }
        if (a.dsum)
#pragma unroll
            for (int v = 0; v < NV; ++v) ds[v].load((const RT *)a.dsum + row * a.ldds, (v * L + lane) * 8, a.cols);
        const float s = a.rstd[row];
        double dot = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * L + lane) * 8;
            dy[v].settle(c, a.cols);
            r[v].settle(c, a.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = dy[v].at(i), n = r[v].at(i) * s;
                dw[v][i] = __builtin_fmaf(d, n, dw[v][i]);
                dot += (double)(d * w[v][i] * n);
            }
            // Where registers are short, the words are kept as they came over the sum (16 bits: 8 registers in place
            // of 24), and dw is done with them (2000 rows of 16 000, bf16: 75 us, 131 from LDS and L2).
            if constexpr (L * NV > 1024) {
                opaque(dw[v]);
                opaque(dy[v].raw);
                opaque(r[v].raw);
            }
        }
        const float mean = (float)(row_sum<L>(dot, sums[turn]) / a.cols);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * L + lane) * 8;
            if (a.dsum) ds[v].settle(c, a.cols);
            float dr[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = dy[v].at(i) * w[v][i], n = r[v].at(i) * s;
                dr[i] = s * (g - n * mean);
                if (a.dsum) dr[i] += ds[v].at(i);
            }
            store_gradients<H, RT, FIT, DROP>(a, gen, row, c, dr);
        }
    }
    if (!a.dW) return;
    float *out = a.ws + blockIdx.x * (int64_t)a.cols;
    if constexpr (PER == 1) {
#pragma unroll
        for (int v = 0; v < NV; ++v) store8<float, FIT>(out, 0, dw[v], (v * L + lane) * 8, a.cols);
    } else {
        // the rows of a wave, then the four waves
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float *to = part + (threadIdx.x >> 6) * (L * NV * 8) + (v * L + lane) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int d = L; d < 64; d <<= 1) dw[v][i] += __shfl_xor(dw[v][i], d);
                if ((threadIdx.x & 63) < L) to[i] = dw[v][i];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < a.cols; c += 256) {
            float x = 0;
#pragma unroll
            for (int g = 0; g < 4; ++g) x += part[g * (L * NV * 8) + c];
            out[c] = x;
        }
    }
}

// Rows that registers do not hold: a workgroup of 1024 goes over each of its rows twice (again from L2) and keeps its
// dw in LDS, or beyond that in the workspace, each thread its own columns.
template <class H, bool DY32, bool R32, bool DROP, bool IN_LDS>
__global__ __launch_bounds__(1024) void rms_norm_backward_long_kernel(NormBackwardArgs a)
{
#pragma clang fp contract(off)
    typedef typename std::conditional<DY32, float, H>::type YT;
    typedef typename std::conditional<R32, float, H>::type RT;
    __shared__ double sums[2][16];
    __shared__ __attribute__((aligned(16))) float held[IN_LDS ? kLong : 4];
    Philox gen;
    if (DROP) gen.init(a.drop);
    float *out = a.dW ? a.ws + blockIdx.x * (int64_t)a.cols : nullptr;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const bool first = row == (int64_t)blockIdx.x, last = row + gridDim.x >= a.rows;
        const float s = a.rstd[row];
        double dot = 0;
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            Eight<YT, kEnds> dy;
            Eight<RT, kEnds> r;
            float w[8], dw[8];
            dy.load((const YT *)a.dY + row * a.lddy, c, a.cols);
            r.load((const RT *)a.r + row * a.ldr, c, a.cols);
            load_weight<H, kEnds>(a.w, a.w32, c, a.cols, w);
            dy.settle(c, a.cols);
            r.settle(c, a.cols);
            if (IN_LDS) {
                *(f32x4 *)dw = *(const f32x4 *)(held + c);
                *(f32x4 *)(dw + 4) = *(const f32x4 *)(held + c + 4);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) dw[i] = out && !first && c + i < a.cols ? out[c + i] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = dy.at(i), n = r.at(i) * s;
                dot += (double)(d * w[i] * n);
                dw[i] = __builtin_fmaf(d, n, first ? 0.0f : dw[i]);
            }
            if (IN_LDS && !last) {
                *(f32x4 *)(held + c) = *(const f32x4 *)dw;
                *(f32x4 *)(held + c + 4) = *(const f32x4 *)(dw + 4);
            } else if (out) {
                store8<float, kEnds>(out, 0, dw, c, a.cols);
            }
        }
        const float mean = (float)(row_sum<1024>(dot, sums[turn]) / a.cols);
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            Eight<YT, kEnds> dy;
            Eight<RT, kEnds> r, ds;
            float w[8], dr[8];
            dy.load((const YT *)a.dY + row * a.lddy, c, a.cols);
            r.load((const RT *)a.r + row * a.ldr, c, a.cols);
            if (a.dsum) ds.load((const RT *)a.dsum + row * a.ldds, c, a.cols);
            load_weight<H, kEnds>(a.w, a.w32, c, a.cols, w);
            dy.settle(c, a.cols);
            r.settle(c, a.cols);
            if (a.dsum) ds.settle(c, a.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = dy.at(i) * w[i], n = r.at(i) * s;
                dr[i] = s * (g - n * mean);
                if (a.dsum) dr[i] += ds.at(i);
            }
            store_gradients<H, RT, kEnds, DROP>(a, gen, row, c, dr);
        }
    }
}

// dw of 16 columns: 64 threads a column over the workspace's rows, then over each other's sums.
template <class H>
__global__ __launch_bounds__(1024) void rms_norm_join_kernel(const float *ws, int groups, int cols, void *dW, bool f32)
{
    __shared__ double part[64][17];
    const int at = threadIdx.x & 15, slice = threadIdx.x >> 4, c = blockIdx.x * 16 + at;
    double x = 0;
    for (int g0 = slice; g0 < groups; g0 += 1024) {       // sixteen loads at once, those outside from inside
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = ws[(int64_t)min(g0 + i * 64, groups - 1) * cols + min(c, cols - 1)];
#pragma unroll
        for (int i = 0; i < 16; ++i) x += g0 + i * 64 < groups ? (double)v[i] : 0.0;
    }
    part[slice][at] = x;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= cols) return;
    x = 0;
    for (int i = 0; i < 64; ++i) x += part[i][at];
    if (f32) ((float *)dW)[c] = (float)x;
    else ((H *)dW)[c] = (H)(float)x;
}

template <class H, bool DY32, bool R32, bool DROP, int L, int NV>
void launch_shape(const NormBackwardArgs &a, int64_t groups, hipStream_t s)
{
    const dim3 g((uint32_t)groups), b(L > 256 ? L : 256);
    const Fit fit = fit_of(a.cols);
    if (fit == kWhole) {
        hipLaunchKernelGGL((rms_norm_backward_kernel<H, DY32, R32, kWhole, DROP, L, NV>), g, b, 0, s, a);
    } else if constexpr (L == 1) {       // rows that end inside a vector have more than eight columns
        hipLaunchKernelGGL((rms_norm_backward_kernel<H, DY32, R32, kTiny, DROP, L, NV>), g, b, 0, s, a);
    } else {
        hipLaunchKernelGGL((rms_norm_backward_kernel<H, DY32, R32, kEnds, DROP, L, NV>), g, b, 0, s, a);
    }
}

template <class H, bool DY32, bool R32, bool DROP>
void launch_cols(const NormBackwardArgs &a, int64_t groups, hipStream_t s)
{
    if (a.cols <= 8) launch_shape<H, DY32, R32, DROP, 1, 1>(a, groups, s);
    else if (a.cols <= 32) launch_shape<H, DY32, R32, DROP, 4, 1>(a, groups, s);
    else if (a.cols <= 64) launch_shape<H, DY32, R32, DROP, 8, 1>(a, groups, s);
    else if (a.cols <= 128) launch_shape<H, DY32, R32, DROP, 16, 1>(a, groups, s);
    else if (a.cols <= 256) launch_shape<H, DY32, R32, DROP, 32, 1>(a, groups, s);
    else if (a.cols <= 512) launch_shape<H, DY32, R32, DROP, 64, 1>(a, groups, s);
    else if (a.cols <= 1024) launch_shape<H, DY32, R32, DROP, 64, 2>(a, groups, s);
    else if (a.cols <= 2048) launch_shape<H, DY32, R32, DROP, 256, 1>(a, groups, s);
    else if (a.cols <= 4096) launch_shape<H, DY32, R32, DROP, 512, 1>(a, groups, s);
    else if (a.cols <= 8192) launch_shape<H, DY32, R32, DROP, 1024, 1>(a, groups, s);
    else if (a.cols <= 16384) launch_shape<H, DY32, R32, DROP, 1024, 2>(a, groups, s);
    else if (a.cols <= kLong) hipLaunchKernelGGL((rms_norm_backward_long_kernel<H, DY32, R32, DROP, true>), dim3((uint32_t)groups), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((rms_norm_backward_long_kernel<H, DY32, R32, DROP, false>), dim3((uint32_t)groups), dim3(1024), 0, s, a);
}

template <class H, bool DY32, bool R32>
void launch_types(const NormBackwardArgs &a, int64_t groups, hipStream_t s)
{
    a.drop.rng ? launch_cols<H, DY32, R32, true>(a, groups, s) : launch_cols<H, DY32, R32, false>(a, groups, s);
}

template <class H>
void launch_half(const NormBackwardArgs &a, int64_t groups, hipStream_t s)
{
    if (a.dy32) a.r32 ? launch_types<H, true, true>(a, groups, s) : launch_types<H, true, false>(a, groups, s);
    else a.r32 ? launch_types<H, false, true>(a, groups, s) : launch_types<H, false, false>(a, groups, s);
}

}  // namespace

size_t rms_norm_backward_workspace(int64_t rows, int32_t cols) { return (size_t)groups_of(rows, cols) * cols * sizeof(float); }

rgnn_status launch_rms_norm_backward(const NormBackwardArgs &a, hipStream_t s)
{
    const int64_t groups = groups_of(a.rows, a.cols);
    if (groups) {
        LaunchScope ls("rms_norm_backward", s);
        if (a.half == RGNN_F16) launch_half<_Float16>(a, groups, s);
        else launch_half<__bf16>(a, groups, s);
    }
    if (a.dW) {
        LaunchScope ls("rms_norm_join", s);
        const dim3 g((uint32_t)((a.cols + 15) / 16));
        if (a.half == RGNN_F16) hipLaunchKernelGGL((rms_norm_join_kernel<_Float16>), g, dim3(1024), 0, s, a.ws, (int)groups, a.cols, a.dW, a.dw32);
        else hipLaunchKernelGGL((rms_norm_join_kernel<__bf16>), g, dim3(1024), 0, s, a.ws, (int)groups, a.cols, a.dW, a.dw32);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "rms_norm_backward launch");
}

}  // namespace rgnn
