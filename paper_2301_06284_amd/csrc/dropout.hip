// dropout.hip -- dropout with the residual's addition, from a counter-based generator: y = [residual +] D(x), and
// its gradient, which is the same of the output's gradient.  No mask is stored.
//
// A workgroup takes a rectangle of rows and vectors of eight columns, up to four vectors a thread.  Bound
// by memory: a value's share of the generator is five 32 x 32 -> 64 products.
#include <algorithm>

#include "rows.h"

namespace rgnn {

namespace {

constexpr int kVectors = 4;

struct Cut {
    int chunks;          // vectors of a row
    int wide, tall;      // a workgroup's: vectors of a row, rows
    int across;          // workgroups side by side
    uint32_t inverse;    // ceil(2^32 / wide)
};

template <class H, bool X32, bool Y32>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, Cut cut)
{
#pragma clang fp contract(off)
    typedef typename std::conditional<X32, float, H>::type XT;
    typedef typename std::conditional<Y32, float, H>::type YT;
    const uint32_t block = flat_block(), down = block / (uint32_t)cut.across;
    const int first = (int)(block - down * cut.across) * cut.wide;
    const int64_t row0 = (int64_t)down * cut.tall;
    Philox gen;
    if (a.drop.rng) gen.init(a.drop);
    Eight<XT> x[kVectors];
    Eight<YT> in[kVectors];
    int64_t row[kVectors];
    int col[kVectors];
#pragma unroll
    for (int u = 0; u < kVectors; ++u) {
        const uint32_t i = threadIdx.x + u * 256;
        const uint32_t r = cut.wide == 1 ? i : __umulhi(i, cut.inverse);
        row[u] = row0 + r;
        col[u] = (first + (int)(i - r * cut.wide)) * 8;
        if ((int)r >= cut.tall || row[u] >= a.rows || col[u] >= a.cols) row[u] = -1;
        if (row[u] < 0) continue;
        x[u].load((const XT *)a.X + row[u] * a.ldx + col[u], a.cols - col[u]);
        if (a.res) in[u].load((const YT *)a.res + row[u] * a.ldr + col[u], a.cols - col[u]);
    }
#pragma unroll
    for (int u = 0; u < kVectors; ++u) {
        if (row[u] < 0) continue;
        float y[8];
        uint32_t word[8];
        if (a.drop.rng) gen.eight(col[u], row[u], word);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float res = a.res ? (float)in[u].v[i] : 0.0f, v = (float)x[u].v[i];
            const float kept = a.res ? __builtin_fmaf(v, a.drop.factor, res) : v * a.drop.factor;
            y[i] = !a.drop.rng || word[i] > a.drop.below ? kept : res;
        }
        store8<YT>(a.Y, row[u] * a.ldy + col[u], y, a.cols - col[u]);
    }
}

template <class H>
void launch_half(const DropoutArgs &a, const Cut &cut, dim3 grid, hipStream_t s)
{
    if (a.x32 && a.y32) hipLaunchKernelGGL((dropout_kernel<H, true, true>), grid, dim3(256), 0, s, a, cut);
    else if (a.x32) hipLaunchKernelGGL((dropout_kernel<H, true, false>), grid, dim3(256), 0, s, a, cut);
    else if (a.y32) hipLaunchKernelGGL((dropout_kernel<H, false, true>), grid, dim3(256), 0, s, a, cut);
    else hipLaunchKernelGGL((dropout_kernel<H, false, false>), grid, dim3(256), 0, s, a, cut);
}

}  // namespace

rgnn_status launch_dropout(const DropoutArgs &a, hipStream_t s)
{
    constexpr int most = 256 * kVectors;
    Cut cut;
    cut.chunks = (a.cols + 7) / 8;
    cut.across = (cut.chunks + most - 1) / most;
    cut.wide = (cut.chunks + cut.across - 1) / cut.across;
    // small matrices: one vector a thread
    const int share = (int64_t)a.rows * cut.chunks <= 256 * 1024 ? 256 : most;
    cut.tall = std::max(1, share / cut.wide);
    cut.inverse = cut.wide == 1 ? 0 : (uint32_t)(((uint64_t(1) << 32) + cut.wide - 1) / cut.wide);
    const int64_t groups = (a.rows + cut.tall - 1) / cut.tall * cut.across;
    if (groups >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many rows");
    {
        LaunchScope ls("dropout", s);
        if (a.half == RGNN_F16) launch_half<_Float16>(a, cut, flat_grid(groups), s);
        else launch_half<__bf16>(a, cut, flat_grid(groups), s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "dropout launch");
}

}  // namespace rgnn
