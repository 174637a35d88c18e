// dropout.hip -- dropout with the residual's addition, from a counter-based generator: y = [residual +] D(x), and
// its gradient, which is the same of the output's gradient.  No mask is stored.
//
// A workgroup takes a rectangle of rows and vectors of eight columns, up to four vectors a thread.  Bound
// by memory: a value's share of the generator is five 32 x 32 -> 64 products.  Measured: 16 384 x 4096 bf16 46 us
// (5.8 TB/s; without dropping 40), with a residual 73 (5.5); 300 007 x 77 fp16 cut out of 101 columns 22 us (4.2); 292 x 64 fp32 2.3 us in a graph.
#include <algorithm>

#include "rows.h"

namespace rgnn {

namespace {

constexpr int kVectors = 4;

struct Cut {
    int wide, tall;      // a workgroup's: vectors of a row, rows
    int across;          // workgroups side by side
    uint32_t inverse;    // ceil(2^32 / wide)
};

// RES: with a residual.  DROP: p is not 0.
template <class H, bool X32, bool Y32, Fit FIT, bool RES, bool DROP>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, Cut cut)
{
#pragma clang fp contract(off)
    typedef typename std::conditional<X32, float, H>::type XT;
    typedef typename std::conditional<Y32, float, H>::type YT;
    const uint32_t block = flat_block(), down = cut.across == 1 ? block : block / (uint32_t)cut.across;
    const int first = (int)(block - down * cut.across) * cut.wide;
    const int64_t row0 = (int64_t)down * cut.tall;
    // Every thread loads all its vectors, those outside from inside: no branch stands between the loads.
    Eight<XT, FIT> x[kVectors];
    Eight<YT, FIT> in[RES ? kVectors : 1];
    int64_t row[kVectors];
    int col[kVectors];
#pragma unroll
    for (int u = 0; u < kVectors; ++u) {
        const uint32_t i = threadIdx.x + u * 256;
        const uint32_t r = cut.wide == 1 ? i : __umulhi(i, cut.inverse);
        row[u] = (int)r < cut.tall ? row0 + r : a.rows;
        col[u] = (first + (int)(i - r * cut.wide)) * 8;
        const int64_t from = min(row[u], a.rows - 1);
        x[u].load((const XT *)a.X + from * a.ldx, col[u], a.cols);
        if constexpr (RES) in[u].load((const YT *)a.res + from * a.ldr, col[u], a.cols);
    }
    Philox gen;
    if constexpr (DROP) gen.init(a.drop);
#pragma unroll
    for (int u = 0; u < kVectors; ++u) {
        if (row[u] >= a.rows || col[u] >= a.cols) continue;
        x[u].settle(col[u], a.cols);
        if constexpr (RES) in[u].settle(col[u], a.cols);
        float y[8];
        uint32_t word[8];
        if constexpr (DROP) gen.eight(col[u], row[u], word);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float res = RES ? in[RES ? u : 0].at(i) : 0.0f, v = x[u].at(i);
            const float kept = RES ? __builtin_fmaf(v, a.drop.factor, res) : v * a.drop.factor;
            y[i] = !DROP || word[i] > a.drop.below ? kept : res;
        }
        store8<YT, FIT>(a.Y, row[u] * a.ldy, y, col[u], a.cols);
    }
}

template <class H, bool X32, bool Y32>
void launch_types(const DropoutArgs &a, const Cut &cut, dim3 grid, hipStream_t s)
{
    auto go = [&](auto fit, auto res, auto drop) {
        hipLaunchKernelGGL((dropout_kernel<H, X32, Y32, decltype(fit)::value, decltype(res)::value, decltype(drop)::value>), grid, dim3(256),
                           0, s, a, cut);
    };
    const std::true_type yes;
    const std::false_type no;
    auto with = [&](auto fit) {
        if (a.drop.rng) a.res ? go(fit, yes, yes) : go(fit, no, yes);
        else a.res ? go(fit, yes, no) : go(fit, no, no);
    };
    const Fit fit = fit_of(a.cols);
    if (fit == kWhole) with(std::integral_constant<Fit, kWhole>());
    else if (fit == kEnds) with(std::integral_constant<Fit, kEnds>());
    else with(std::integral_constant<Fit, kTiny>());
}

// Of calls with a 16-bit type.
template <class H>
void launch_half(const DropoutArgs &a, const Cut &cut, dim3 grid, hipStream_t s)
{
    if (a.x32) launch_types<H, true, false>(a, cut, grid, s);
    else a.y32 ? launch_types<H, false, true>(a, cut, grid, s) : launch_types<H, false, false>(a, cut, grid, s);
}

}  // namespace

rgnn_status launch_dropout(const DropoutArgs &a, hipStream_t s)
{
    constexpr int most = 256 * kVectors;
    const int chunks = (a.cols + 7) / 8;          // vectors of a row
    Cut cut;
    cut.across = (chunks + most - 1) / most;
    cut.wide = (chunks + cut.across - 1) / cut.across;
    // small matrices: one vector a thread
    const int share = (int64_t)a.rows * chunks <= 256 * 1024 ? 256 : most;
    cut.tall = std::max(1, share / cut.wide);
    cut.inverse = cut.wide == 1 ? 0 : (uint32_t)(((uint64_t(1) << 32) + cut.wide - 1) / cut.wide);
    const int64_t groups = (a.rows + cut.tall - 1) / cut.tall * cut.across;
    if (groups >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many rows");
    {
        LaunchScope ls("dropout", s);
        if (a.x32 && a.y32) launch_types<__bf16, true, true>(a, cut, flat_grid(groups), s);
        else if (a.half == RGNN_F16) launch_half<_Float16>(a, cut, flat_grid(groups), s);
        else launch_half<__bf16>(a, cut, flat_grid(groups), s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "dropout launch");
}

}  // namespace rgnn
