// rms_norm.hip -- root-mean-square norm of rows with the residual's addition and dropout:
// r = round(residual + D(x)), s = 1 / sqrt(mean(r^2) + eps), y = (r s) w, as rows or as 8-bit codes.
//
// A row is read once and stays in registers from its loads to its stores: a few lanes of a wave hold a short row, a wave
// or a workgroup a long one, eight columns a lane at a time.  Squares are summed in 64 bits, which costs
// next to nothing where memory is waited for (16 384 x 2048 74.4 us, in 32 bits 74.3; 8000 x 4096 42.8 and 42.5; 600 000 x 24
// 30.8 and 28.5).  A sum is off by some 2^-53 of itself, so that 1 / rms is the formula's to half a step of fp32, and rows
// that are cut in another way differ only where theirs lies next to a border of that rounding.
//
// Bound by memory, a few rows by the launch.  Measured, with residual and sum: 1 000 003 x 64 fp32 181 us (5.7 TB/s), 16 384 x
// 2048 bf16 with an fp32 residual and dropout 74 us (5.4), 8192 x 4096 bf16 into e4m3 45 us (5.2), 15 000 x 2048 bf16
// 37 to 39 us (6.3, from the last-level cache in part), 10 007 x 333 fp16 9.4 us (8.7 in a graph), 8 x 2048 2.9 us in a graph.
#include <algorithm>

#include "rows.h"

namespace rgnn {

namespace {

// r of eight columns: the sum in fp32, the kept value's product not rounded before it, rounded to r's type.
template <class RT>
__device__ __forceinline__ void sum8(const NormArgs &a, const Philox &gen, int64_t row, int col, const float (&x)[8], const float (&res)[8],
                                     float (&r)[8])
{
    if (a.drop.rng) {
        uint32_t word[8];
        gen.eight(col, row, word);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = word[i] > a.drop.below ? __builtin_fmaf(x[i], a.drop.factor, res[i]) : res[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = x[i] + res[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (float)(RT)r[i];
}

// What lies beyond fp32 counts as its largest number, so that zeros times it are zeros for any eps > 0; of a row of zeros
// without eps it is infinite.
__device__ __forceinline__ float inverse_rms(double squares, int cols, double eps)
{
    const double s = 1.0 / sqrt(squares / cols + eps);
    return s < __builtin_inf() ? (float)fmin(s, 0x1.fffffep+127) : (float)s;
}

// L threads hold a row, NV vectors of eight columns each.
template <class H, bool X32, bool R32, Fit FIT, int L, int NV>
__global__ __launch_bounds__(L > 64 ? L : 256) void rms_norm_kernel(NormArgs a)
{
#pragma clang fp contract(off)
    typedef typename std::conditional<X32, float, H>::type XT;
    typedef typename std::conditional<R32, float, H>::type RT;
    constexpr int PER = L > 64 ? 1 : 256 / L;       // rows of a workgroup
    __shared__ double sums[L > 64 ? L / 64 : 1];
    __shared__ uint32_t tops[L > 64 ? L / 64 : 1];
    const int64_t row = flat_block() * (int64_t)PER + (PER > 1 ? threadIdx.x / L : 0);
    if (row >= a.rows) return;                       // all lanes of a row
    const int lane = threadIdx.x % L;

    Eight<XT, FIT> x[NV];
    Eight<RT, FIT> in[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * L + lane) * 8;
        x[v].load((const XT *)a.X + row * a.ldx, c, a.cols);
    }
    if (a.res)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * L + lane) * 8;
            in[v].load((const RT *)a.res + row * a.ldr, c, a.cols);
        }
    Philox gen;
    if (a.drop.rng) gen.init(a.drop);
    float r[NV][8], w[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) load_weight<H, FIT>(a.w, a.w32, (v * L + lane) * 8, a.cols, w[v]);
    double squares = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = (v * L + lane) * 8;
        float f[8], res[8];
        x[v].settle(c, a.cols);
        if (a.res) in[v].settle(c, a.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[i] = x[v].at(i);
            res[i] = a.res ? in[v].at(i) : 0.0f;
        }
        sum8<RT>(a, gen, row, c, f, res, r[v]);
        if (a.sum) store8<RT, FIT>(a.sum, row * a.lds, r[v], c, a.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) squares = __builtin_fma((double)r[v][i], (double)r[v][i], squares);
    }
    const float s = inverse_rms(row_sum<L>(squares, sums), a.cols, a.eps);
    if (a.rstd && lane == 0) a.rstd[row] = s;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) r[v][i] = r[v][i] * s * w[v][i];

    if (a.out <= kRowsF32) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * L + lane) * 8;
            if (a.out == kRowsF32) store8<float, FIT>(a.Y, row * a.ldy, r[v], c, a.cols);
            else store8<H, FIT>(a.Y, row * a.ldy, r[v], c, a.cols);
        }
        return;
    }
    if constexpr (L >= 16) {      // codes: what lies behind the columns is zero up to whole blocks of 128, 16 lanes or more
        const int kp = fp8_width(a.cols);
        uint8_t *codes = (uint8_t *)a.Y + row * kp;
        if (a.out == kRowsE4m3) {
            const int ks = fp8_scales(a.cols);
            uint8_t *sc = (uint8_t *)a.scales + row * ks;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c = (v * L + lane) * 8;
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, c + i < a.cols ? magnitude_bits(r[v][i]) : 0);
                const int byte = e4m3_scale_byte(lanes_max<16>(top));
#pragma unroll
                for (int i = 0; i < 8; ++i) r[v][i] = c + i < a.cols ? r[v][i] : 0.0f;
                if (c < kp) store_e4m3(codes + c, r[v], byte);
                if (c < kp && (lane & 15) == 0) sc[c >> 7] = (uint8_t)byte;
            }
            if (lane < ks - (kp >> 7)) sc[(kp >> 7) + lane] = 127;
            return;
        }
        uint32_t top = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, (v * L + lane) * 8 + i < a.cols ? magnitude_bits(r[v][i]) : 0);
        const float scale = int8_scale(row_max<L>(top, tops)), inverse = 1.0f / scale;
        if (lane == 0) ((float *)a.scales)[row] = scale;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = (v * L + lane) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[v][i] = c + i < a.cols ? r[v][i] : 0.0f;
            if (c < kp) store_int8(codes + c, r[v], inverse, scale != scale);
        }
    }
}

// Rows that registers do not hold: a workgroup of 1024 goes over its row once for the sum, again for the
// outputs and, with 8-bit integers, in between for the largest.  What it reads again is what it stored (the sum), or the
// inputs where no sum is kept.
template <class H, bool X32, bool R32>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(NormArgs a)
{
#pragma clang fp contract(off)
    typedef typename std::conditional<X32, float, H>::type XT;
    typedef typename std::conditional<R32, float, H>::type RT;
    __shared__ double sums[16];
    __shared__ uint32_t tops[16];
    const int64_t row = flat_block();
    if (row >= a.rows) return;
    const int kp = a.out <= kRowsF32 ? a.cols : fp8_width(a.cols);
    Philox gen;
    if (a.drop.rng) gen.init(a.drop);
    auto sum = [&](int c, float (&r)[8]) {
        Eight<XT, kEnds> x;
        Eight<RT, kEnds> in;
        x.load((const XT *)a.X + row * a.ldx, c, a.cols);
        if (a.res) in.load((const RT *)a.res + row * a.ldr, c, a.cols);
        x.settle(c, a.cols);
        if (a.res) in.settle(c, a.cols);
        float f[8], res[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[i] = x.at(i);
            res[i] = a.res ? in.at(i) : 0.0f;
        }
        sum8<RT>(a, gen, row, c, f, res, r);
    };
    auto again = [&](int c, float s, float (&y)[8]) {       // the norm's output in fp32, zero behind the columns
        float w[8];
        if (a.sum) {
            Eight<RT, kEnds> in;
            in.load((const RT *)a.sum + row * a.lds, c, a.cols);
            in.settle(c, a.cols);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = in.at(i);
        } else {
            sum(c, y);
        }
        load_weight<H, kEnds>(a.w, a.w32, c, a.cols, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = c + i < a.cols ? y[i] * s * w[i] : 0.0f;
    };
    double squares = 0;
    for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
        float r[8];
        sum(c, r);
        if (a.sum) store8<RT, kEnds>(a.sum, row * a.lds, r, c, a.cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) squares = __builtin_fma((double)r[i], (double)r[i], squares);
    }
    const float s = inverse_rms(row_sum<1024>(squares, sums), a.cols, a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = s;
    float scale = 0;
    if (a.out == kRowsInt8) {
        uint32_t top = 0;
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            float y[8];
            again(c, s, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(y[i]));
        }
        scale = int8_scale(row_max<1024>(top, tops));
        if (threadIdx.x == 0) ((float *)a.scales)[row] = scale;
    }
    const float inverse = 1.0f / scale;
    uint8_t *codes = (uint8_t *)a.Y + row * kp;
    uint8_t *sc = (uint8_t *)a.scales + row * fp8_scales(a.cols);
    for (int c = threadIdx.x * 8; c < kp; c += 8192) {
        float y[8];
        again(c, s, y);
        if (a.out == kRowsHalf) store8<H, kEnds>(a.Y, row * a.ldy, y, c, a.cols);
        else if (a.out == kRowsF32) store8<float, kEnds>(a.Y, row * a.ldy, y, c, a.cols);
        else if (a.out == kRowsInt8) store_int8(codes + c, y, inverse, scale != scale);
        else {      // kp is whole blocks: the 16 lanes of a block are here together
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(y[i]));
            const int byte = e4m3_scale_byte(lanes_max<16>(top));
            store_e4m3(codes + c, y, byte);
            if ((threadIdx.x & 15) == 0) sc[c >> 7] = (uint8_t)byte;
        }
    }
    if (a.out == kRowsE4m3 && (int)threadIdx.x < fp8_scales(a.cols) - (kp >> 7)) sc[(kp >> 7) + threadIdx.x] = 127;
}

template <class H, bool X32, bool R32, Fit FIT, int L, int NV>
void launch_rows(const NormArgs &a, hipStream_t s)
{
    constexpr int PER = L > 64 ? 1 : 256 / L;
    hipLaunchKernelGGL((rms_norm_kernel<H, X32, R32, FIT, L, NV>), flat_grid((a.rows + PER - 1) / PER), dim3(L > 64 ? L : 256), 0, s, a);
}

// The threads of a row: as many as it has vectors of eight, a power of two, which measured faster than fewer threads with
// several vectors (bf16, with residual and sum: 60 000 x 512 64 threads 39.2 us, 32 of two 43.2; 30 000 x 1000 128 threads
// 41.4, 64 of two 42.8; 600 000 x 24 fp16 4 lanes 23.3, 8 34.4; 8000 x 4096 512 threads 41.9, 256 of two 43.4; 4000 x 8192 1024 threads 44.0, 256 of four 48.5; 8 x 1000
// 2.6 and 3.2).  Two vectors a thread for many rows that end inside one (80 000 x 333 45.2 us, 64 threads 46.3; 30 000 x 1001
// 40.5, 128 threads 46.7; but 1000 x 333 3.6 and 2.8) and for long rows of codes (4000 x 8192 into int8 42.4, 1024 threads 44.6).
template <class H, bool X32, bool R32, Fit FIT>
void launch_cols(const NormArgs &a, hipStream_t s)
{
    const bool codes = a.out > kRowsF32;
    const int cols = codes ? fp8_width(a.cols) : a.cols;
    if constexpr (FIT == kEnds)
        if (a.rows > 4096 && cols > 256 && cols <= 1024)
            return cols <= 512 ? launch_rows<H, X32, R32, FIT, 32, 2>(a, s) : launch_rows<H, X32, R32, FIT, 64, 2>(a, s);
    if constexpr (FIT == kWhole)      // rows that end inside a vector have more than eight columns
        if (cols <= 8) return launch_rows<H, X32, R32, FIT, 1, 1>(a, s);
    if (cols <= 32) launch_rows<H, X32, R32, FIT, 4, 1>(a, s);
    else if (cols <= 64) launch_rows<H, X32, R32, FIT, 8, 1>(a, s);
    else if (cols <= 128) launch_rows<H, X32, R32, FIT, 16, 1>(a, s);
    else if (cols <= 256) launch_rows<H, X32, R32, FIT, 32, 1>(a, s);
    else if (cols <= 512) launch_rows<H, X32, R32, FIT, 64, 1>(a, s);
    else if (cols <= 1024) launch_rows<H, X32, R32, FIT, 128, 1>(a, s);
    else if (cols <= 2048) launch_rows<H, X32, R32, FIT, 256, 1>(a, s);
    else if (cols <= 4096) launch_rows<H, X32, R32, FIT, 512, 1>(a, s);
    else if (cols <= 8192 && !codes) launch_rows<H, X32, R32, FIT, 1024, 1>(a, s);
    else if (cols <= 8192) launch_rows<H, X32, R32, FIT, 512, 2>(a, s);
    else if (cols <= 16384) launch_rows<H, X32, R32, FIT, 1024, 2>(a, s);
    else if (cols <= 32768) launch_rows<H, X32, R32, FIT, 1024, 4>(a, s);
    else hipLaunchKernelGGL((rms_norm_long_kernel<H, X32, R32>), flat_grid(a.rows), dim3(1024), 0, s, a);
}

template <class H, bool X32, bool R32>
void launch_types(const NormArgs &a, hipStream_t s)
{
    const Fit fit = fit_of(a.cols);
    if (fit == kWhole) launch_cols<H, X32, R32, kWhole>(a, s);
    else if (fit == kEnds) launch_cols<H, X32, R32, kEnds>(a, s);
    else if (a.out <= kRowsF32) launch_rows<H, X32, R32, kTiny, 1, 1>(a, s);
    else launch_rows<H, X32, R32, kTiny, 16, 1>(a, s);
}

template <class H>
void launch_half(const NormArgs &a, hipStream_t s)
{
    if (a.x32) return a.r32 ? launch_types<H, true, true>(a, s) : launch_types<H, true, false>(a, s);
    return a.r32 ? launch_types<H, false, true>(a, s) : launch_types<H, false, false>(a, s);
}

}  // namespace

rgnn_status launch_rms_norm(const NormArgs &a, hipStream_t s)
{
    {
        LaunchScope ls("rms_norm", s);
        if (a.half == RGNN_F16) launch_half<_Float16>(a, s);
        else launch_half<__bf16>(a, s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "rms_norm launch");
}

}  // namespace rgnn
