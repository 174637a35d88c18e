// typed_wgrad.hip -- the weight gradient of the typed linear over ragged segments,
// dW[t] = sum over the positions i of type t of X[gather[i]]^T dY[dy_gather[i]].
//
// A workgroup takes BK x BN values of one type's gradient and walks the type's positions in
// steps of 64 (fp32: 32), a row of X and of dY each, straight from memory to LDS, the next
// step while this one is multiplied.  Both operands have the contraction across the rows,
// so 16-bit fragments are read with the transposing LDS read (the layout of "rows of n" in
// typed_linear.hip).
//
// A type with more positions than a piece (WgradPlan) is cut into pieces whose sums, in
// fp32, go through the workspace and are added in ascending order by a second kernel: no
// atomics, the same result every time.
//
// What bounds it, and what it measured: memory at narrow widths (300 007 rows, 64 x 64, fp16: 17 us, 4.5
// TB/s, and 7 us for the join), the matrix cores and the gradients' bytes at wide ones (8192 rows of 16
// types, 2048 x 1536, bf16: 87 us, 0.59 PFLOP/s and 100 MB written; tiles of different types take as
// different times as these have rows), launches below (10 007 rows, 100 x 77, fp32: 13 us and 4).
#include <algorithm>

#include "wide_tile.h"

namespace rgnn {

namespace {

// Pieces of a type's rows: one up to `whole` of them, of `chunk` rows beyond; and those whose sums
// go through the workspace.
struct Cut {
    int64_t whole, chunk;
    __device__ __forceinline__ bool split(int64_t rows) const { return rows > whole; }
    __device__ __forceinline__ int64_t pieces(int64_t rows) const { return split(rows) ? (rows + chunk - 1) / chunk : 1; }
    __device__ __forceinline__ int64_t slots(int64_t rows) const { return split(rows) ? (rows + chunk - 1) / chunk : 0; }
};

struct WgradK {
    const char *X, *dY;
    int64_t x_rows, ldx, dy_rows, lddy;   // ld in bytes
    const int32_t *gather, *dy_gather;
    const int64_t *ptr;
    int T;
    int64_t M;
    int K, N;
    void *dW;
    int f32;                     // fp32 gradients
    const char *x_end, *dy_end;  // behind the last element
    Cut cut;
    int64_t slots;
    float *partial;
    int window;
};

// One operand's loads: rows of the contraction, B columns from c0 on.  A position whose row of
// either operand lies outside its matrix brings zeros for both: nothing, whatever the other holds.
template <class T, int B, int NW>
struct Side {
    typedef typename T::elem E;
    static constexpr int KE = 128 / sizeof(E), L = B / 8 / NW, CH = B * sizeof(E) / 16, UC = sizeof(E) == 4 ? 4 : 2;
    static_assert(L * 8 * NW == B, "whole loads");
    const char *base;
    const int32_t *index, *other;         // other: the other operand's
    int64_t rows, other_rows, ld, pos, end;   // pos: the position of this lane's first load of the next step
    int col[L];                  // bytes
    int next[L];                 // with index arrays: the next step's rows, -1 for zeros
    int wave;

    __device__ __forceinline__ static int row_of(int x, int wave, int lane) { return ((x * NW + wave) * 64 + lane) / CH; }

    __device__ __forceinline__ void init(const char *m, const int32_t *idx, int64_t m_rows, const int32_t *other_idx, int64_t o_rows,
                                         int64_t m_ld, int64_t p0, int64_t p1, int c0, int width, int w, int lane)
    {
        base = m; index = idx; rows = m_rows; other = other_idx; other_rows = o_rows; ld = m_ld; pos = p0; end = p1; wave = w;
#pragma unroll
        for (int x = 0; x < L; ++x) {
            const int at = (x * NW + w) * 64 + lane, k = at / CH, p = at % CH;
            const int c = ((p / UC) ^ unit_turn<T, B>(k)) * UC + p % UC;
            const int j = c0 + c * (16 / (int)sizeof(E));
            col[x] = (j < width ? j : 0) * (int)sizeof(E);
        }
        fetch(lane);
    }
    __device__ __forceinline__ void fetch(int lane)
    {
        if (!index && !other) return;
#pragma unroll
        for (int x = 0; x < L; ++x) {
            const int64_t i = pos + row_of(x, wave, lane);
            int r = -1;
            if (i < end) {
                r = index ? index[i] : (int)i;
                if (r >= rows) r = -1;
                const int o = other ? other[i] : 0;
                if (o < 0 || (other && o >= other_rows)) r = -1;
            }
            next[x] = r;
        }
    }
    // the row of load x, or one below 0
    __device__ __forceinline__ int64_t row_at(int x, int lane) const
    {
        if (index || other) return next[x];
        const int64_t i = pos + row_of(x, wave, lane);
        return i < end ? i : -1;
    }
    // rows on any address: a step's loads into registers, and from there to LDS
    __device__ __forceinline__ void take(i32x4 (&r)[L], const char *last, int lane)
    {
#pragma unroll
        for (int x = 0; x < L; ++x) {
            const int64_t row = row_at(x, lane);
            r[x] = row >= 0 ? load_any<E>(base + row * ld + col[x], last) : i32x4{0, 0, 0, 0};
        }
        pos += KE;
        fetch(lane);
    }
    __device__ __forceinline__ void put(const i32x4 (&r)[L], char *lds, int lane) const
    {
#pragma unroll
        for (int x = 0; x < L; ++x) *(i32x4 *)(lds + (x * NW + wave) * 1024 + lane * 16) = r[x];
    }
    __device__ __forceinline__ void load(char *lds, int lane)
    {
#pragma unroll
        for (int x = 0; x < L; ++x) {
            const int64_t row = row_at(x, lane);
            load_lds(row >= 0 ? base + row * ld + col[x] : (const char *)&kZeros, lds + (x * NW + wave) * 1024);
        }
        pos += KE;
        fetch(lane);
    }
};

// ANY: rows on any address (typed_linear.hip).  Two waves a SIMD, so that sums stay in the registers that the
// compiler would else copy them to and from.
template <class T, int BK, int BN, int WM, int WN, bool ANY>
__global__ __launch_bounds__(WM *WN * 64, 2) void typed_wgrad_kernel(WgradK a)
{
    typedef typename T::elem E;
    constexpr int NW = WM * WN, KE = 128 / sizeof(E);
    constexpr int FM = BK / WM / 16, FN = BN / WN / 16;
    __shared__ __attribute__((aligned(1024))) char sx0[BK * 128], sy0[BN * 128], sx1[BK * 128], sy1[BN * 128];

    const int nk = (a.K + BK - 1) / BK, nn = (a.N + BN - 1) / BN, per = nk * nn;
    const Cut cut = a.cut;
    Piece p;
    if (!find_piece(a.ptr, a.T, a.M, xcd_tile(a.window), [=](int64_t c) { return cut.pieces(c) * per; },
                    [=](int64_t c) { return cut.slots(c); }, p))
        return;
    const bool split = cut.split(p.end - p.begin);
    const int part = (int)(p.index / per);
    int ki, ni;
    tile_place((int)(p.index - (int64_t)part * per), nk, nn, ki, ni);
    const int64_t p0 = p.begin + part * cut.chunk;
    const int64_t p1 = split ? min(p0 + cut.chunk, p.end) : p.end;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4, wm = wave / WN, wn = wave % WN;

    Side<T, BK, NW> x;
    Side<T, BN, NW> y;
    x.init(a.X, a.gather, a.x_rows, a.dy_gather, a.dy_rows, a.ldx, p0, p1, ki * BK, a.K, wave, lane);
    y.init(a.dY, a.dy_gather, a.dy_rows, a.gather, a.x_rows, a.lddy, p0, p1, ni * BN, a.N, wave, lane);

    // fragment f lies at (units before the wave's) + (f ^ turn): the turn sits in the address
    // bits of the units, so an exclusive or with f's bits moves from fragment to fragment
    constexpr int UB = sizeof(E) == 2 ? 32 : 64;
    const int kr = sizeof(E) == 2 ? g * 8 + (r16 >> 2) : g * 4, in = sizeof(E) == 2 ? (r16 & 3) * 8 : r16 * 4;
    static_assert((FM & (FM - 1)) == 0 && (FN & (FN - 1)) == 0, "powers of two");
    int xat = (kr * BK * (int)sizeof(E) + in) | ((wm * FM) ^ unit_turn<T, BK>(kr)) * UB;
    int yat = (kr * BN * (int)sizeof(E) + in) | ((wn * FN) ^ unit_turn<T, BN>(kr)) * UB;
    f32x4 acc[FM][FN] = {};
    auto fragment = [&](const char *lds, int off, int q, int width) -> i32x4 {
        if constexpr (sizeof(E) == 2) {
            const uint64_t u = read_turned(lds + off + q * 32 * width * 2), v = read_turned(lds + off + (q * 32 + 4) * width * 2);
            return i32x4{(int)u, (int)(u >> 32), (int)v, (int)(v >> 32)};
        } else {
            i32x4 r;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = *(const int *)(lds + off + (q * 16 + i) * width * 4);
            return r;
        }
    };
    auto multiply = [&](const char *sx, const char *sy) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" : "+v"(xat), "+v"(yat));   // the fragments' addresses are made here, not kept in registers
            i32x4 fx[FM], fy[FN];
#pragma unroll
            for (int f = 0; f < FN; ++f) fy[f] = fragment(sy, yat ^ f * UB, q, BN);
#pragma unroll
            for (int f = 0; f < FM; ++f) fx[f] = fragment(sx, xat ^ f * UB, q, BK);
#pragma unroll
            for (int m = 0; m < FM; ++m)
#pragma unroll
                for (int f = 0; f < FN; ++f) acc[m][f] = mma16<T>(fy[f], fx[m], acc[m][f]);
        }
    };

    const int steps = (int)((p1 - p0 + KE - 1) / KE);
    int step = 0;
    if constexpr (ANY) {
        i32x4 rx[Side<T, BK, NW>::L], ry[Side<T, BN, NW>::L];
        auto take = [&]() {
            x.take(rx, a.x_end, lane);
            y.take(ry, a.dy_end, lane);
        };
        auto put = [&](char *lx, char *ly) {
            x.put(rx, lx, lane);
            y.put(ry, ly, lane);
        };
        if (steps > 0) {
            take();
            put(sx0, sy0);
            if (steps > 1) take();
        }
        for (; step + 2 <= steps; step += 2) {
            __syncthreads();
            multiply(sx0, sy0);
            put(sx1, sy1);
            if (step + 2 < steps) take();
            __syncthreads();
            multiply(sx1, sy1);
            if (step + 2 < steps) put(sx0, sy0);
            if (step + 3 < steps) take();
        }
        if (step < steps) {
            __syncthreads();
            multiply(sx0, sy0);
        }
    } else {
        if (steps > 0) {
            x.load(sx0, lane);
            y.load(sy0, lane);
        }
        for (; step + 2 <= steps; step += 2) {
            step_barrier<0>();
            x.load(sx1, lane);
            y.load(sy1, lane);
            multiply(sx0, sy0);
            step_barrier<0>();
            if (step + 2 < steps) {
                x.load(sx0, lane);
                y.load(sy0, lane);
            }
            multiply(sx1, sy1);
        }
        if (step < steps) {
            step_barrier<0>();
            multiply(sx0, sy0);
        }
    }

    const int64_t slot = p.before + part;
    const int64_t at0 = (split ? slot : (int64_t)p.type) * a.K;
#pragma unroll
    for (int m = 0; m < FM; ++m) {
        const int k = ki * BK + (wm * FM + m) * 16 + r16;
        if (k >= a.K) continue;
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            const int n = ni * BN + (wn * FN + f) * 16 + g * 4;
            if (n >= a.N) continue;
            const int64_t at = (at0 + k) * a.N + n;
            if (split) write4(a.partial + at, acc[m][f], a.N - n);
            else if (sizeof(E) == 4 || a.f32) write4((float *)a.dW + at, acc[m][f], a.N - n);
            else write4((E *)a.dW + at, acc[m][f], a.N - n);
        }
    }
}

// The wide tile (wide_tile.h): rows as they are (without index arrays), whose places a base for
// all lanes and an offset for each tell.
template <class T>
__global__ __launch_bounds__(256, 1) void typed_wgrad_wide_kernel(WgradK a)
{
    typedef typename T::elem E;
    constexpr int KE = kWideKB / sizeof(E);
    __shared__ __attribute__((aligned(1024))) char s0[2 * kWideStage], s1[2 * kWideStage], s2[2 * kWideStage], s3[2 * kWideStage];
    __shared__ int to[kWide];
    char *a0 = s0, *b0 = s0 + kWideStage, *a1 = s1, *b1 = s1 + kWideStage;
    char *a2 = s2, *b2 = s2 + kWideStage, *a3 = s3, *b3 = s3 + kWideStage;

    const int nk = (a.K + kWide - 1) / kWide, nn = (a.N + kWide - 1) / kWide, per = nk * nn;
    const Cut cut = a.cut;
    Piece p;
    if (!find_piece(a.ptr, a.T, a.M, xcd_tile(a.window), [=](int64_t c) { return cut.pieces(c) * per; },
                    [=](int64_t c) { return cut.slots(c); }, p))
        return;
    const bool split = cut.split(p.end - p.begin);
    const int part = p.index / per;
    int ki, ni;
    tile_place(p.index - part * per, nk, nn, ki, ni);
    const int64_t p0 = p.begin + part * cut.chunk;
    const int rows = (int)(split ? min(cut.chunk, p.end - p0) : p.end - p0);
    const int k0 = ki * kWide, n0 = ni * kWide;
    const int64_t slot = p.before + part;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    to[threadIdx.x] = k0 + (int)threadIdx.x < a.K ? (int)threadIdx.x : -1;

    WideSide sx, sy;
    sx.base = a.X + p0 * a.ldx + k0 * (int64_t)sizeof(E);
    sy.base = a.dY + p0 * a.lddy + n0 * (int64_t)sizeof(E);
    sx.step = KE * a.ldx;
    sy.step = KE * a.lddy;
    const int row0 = wave * 2 + (lane >> 5);         // of a step's 32, and 8 x more for load x
#pragma unroll
    for (int x = 0; x < kWideLoads; ++x) {
        const int k = row0 + x * 8, pos = lane & 31, j = ((pos >> 1 ^ wide_turn_n(k)) * 2 + (pos & 1)) * 8;
        sx.off[x] = (uint32_t)(k * a.ldx) + (k0 + j < a.K ? j : 0) * (uint32_t)sizeof(E);
        sy.off[x] = (uint32_t)(k * a.lddy) + (n0 + j < a.N ? j : 0) * (uint32_t)sizeof(E);
    }
    const int whole = rows / KE, steps = (rows + KE - 1) / KE;
    WideFragments<true> fx, fy;
    fx.init(wm * 128, lane);
    fy.init(wn * 128, lane);

    f32x16 acc[4][4] = {};
    constexpr int LOADS = 2 * kWideLoads;
    auto load = [&](char *ta, char *tb) {
        sx.load<kWideLoads>(ta, wave);
        sy.load<kWideLoads>(tb, wave);
        sx.base += sx.step;
        sy.base += sy.step;
    };
    auto edge = [&](char *ta, char *tb, int step) {
        if (step < whole) return load(ta, tb);
        auto in = [&](int x) { return step * KE + row0 + x * 8 < rows; };
        sx.load_edge<kWideLoads>(ta, wave, in);
        sy.load_edge<kWideLoads>(tb, wave, in);
    };
    auto multiply = [&](const i32x8 (&x)[4], const i32x8 (&y)[4], f32x16 (&c)[4][4]) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n) c[m][n] = mma32<T>(chunk_of(y[n], q), chunk_of(x[m], q), c[m][n]);
    };
    // a type without rows: nothing to walk, zeros to write
    if (steps > 0) wide_walk<4, true, true, LOADS>(a0, b0, a1, b1, a2, b2, a3, b3, fx, fy, steps, whole, load, edge, multiply, [](int) {}, acc);
    else __syncthreads();

    const int64_t at0 = (split ? slot : (int64_t)p.type) * a.K + k0;
    if (!split && !a.f32) {
        char *mine = wave == 0 ? s0 : wave == 1 ? s1 : wave == 2 ? s2 : s3;
        wide_write<E, 4>(mine, acc, (E *)a.dW + at0 * a.N + n0 + wn * 128, a.N, a.N - n0 - wn * 128, lane, to + wm * 128);
        return;
    }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int k = wm * 128 + m * 32 + (lane & 31);
        if (k0 + k >= a.K) continue;
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = n0 + wn * 128 + n * 32 + q * 8 + (lane >> 5) * 4;
                if (j >= a.N) continue;
                const int64_t at = (at0 + k) * a.N + j;
                const f32x4 v = {acc[m][n][q * 4], acc[m][n][q * 4 + 1], acc[m][n][q * 4 + 2], acc[m][n][q * 4 + 3]};
                if (split) write4(a.partial + at, v, a.N - j);
                else write4((float *)a.dW + at, v, a.N - j);
            }
    }
}

// dW[t] of the types with several pieces.  A workgroup takes 64 V values of one type's gradient
// at a time and adds a quarter of the pieces in each wave, then the quarters.
template <class E, int V>
__global__ __launch_bounds__(256) void wgrad_join_kernel(const int64_t *ptr, int T, int64_t M, Cut cut, int64_t KN,
                                                         const float *partial, void *dW, int out_f32)
{
    typedef float vec __attribute__((ext_vector_type(V)));
    __shared__ vec sums[4][64];
    Piece p;
    if (!find_piece(ptr, T, M, blockIdx.y, [](int64_t) { return 1; }, [=](int64_t c) { return cut.slots(c); }, p)) return;
    const int64_t n = cut.slots(p.end - p.begin);
    if (n == 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t quarter = (n + 3) / 4, c0 = min(wave * quarter, n), c1 = min(c0 + quarter, n);
    for (int64_t i0 = blockIdx.x * (int64_t)(64 * V); i0 < KN; i0 += (int64_t)gridDim.x * (64 * V)) {
        const int64_t i = i0 + lane * V;
        vec s = 0.0f;
        if (i < KN) {
            const float *x = partial + p.before * KN + i;
#pragma unroll 4
            for (int64_t c = c0; c < c1; ++c) s += *(const vec *)(x + c * KN);
        }
        sums[wave][lane] = s;
        __syncthreads();
        if (wave == 0 && i < KN) {
            s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
            const int64_t at = p.type * KN + i;
#pragma unroll
            for (int q = 0; q < V; ++q) {
                if (out_f32) ((float *)dW)[at + q] = s[q];
                else ((E *)dW)[at + q] = (E)s[q];
            }
        }
        __syncthreads();
    }
}

template <class E>
void launch_join(const WgradArgs &a, const WgradPlan &plan, hipStream_t s)
{
    const int64_t kn = (int64_t)a.K * a.N;
    const int v = kn % 4 == 0 ? 4 : 1;
    // a workgroup looks for its type first: no more than fill the chip (16 types, 2048 x 1536: 1024 of them
    // 5.5 us, 4096 6.7), but 16 for a type while all are a few thousand (96 types, 64 x 64: 7.2 us, 10 for each 9.6)
    const int64_t most = std::max<int64_t>(1, std::max<int64_t>(1024 / a.T, std::min<int64_t>(16, 4096 / a.T)));
    const dim3 g((uint32_t)std::min((kn + 64 * v - 1) / (64 * v), most), (uint32_t)a.T);
    const int f32 = a.dw_dtype == RGNN_F32;
    const float *part = (const float *)a.ws;
    LaunchScope ls("typed_wgrad_join", s);
    if (v == 4) hipLaunchKernelGGL((wgrad_join_kernel<E, 4>), g, dim3(256), 0, s, a.type_ptr, a.T, a.M, Cut{plan.whole, plan.chunk}, kn, part, a.dW, f32);
    else hipLaunchKernelGGL((wgrad_join_kernel<E, 1>), g, dim3(256), 0, s, a.type_ptr, a.T, a.M, Cut{plan.whole, plan.chunk}, kn, part, a.dW, f32);
}

template <class T, int BK, int BN, int WM, int WN, bool ANY>
rgnn_status launch_tile(WgradK k, hipStream_t s)
{
    const int64_t tiles = (k.T + k.slots) * ((k.K + BK - 1) / BK) * ((k.N + BN - 1) / BN);
    k.window = xcd_window(tiles);
    const int64_t grid = xcd_grid(tiles, k.window);
    if (grid >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many tiles");
    hipLaunchKernelGGL((typed_wgrad_kernel<T, BK, BN, WM, WN, ANY>), flat_grid(grid), dim3(WM * WN * 64), 0, s, k);
    return RGNN_OK;
}

template <class T>
rgnn_status launch_wide(WgradK k, hipStream_t s)
{
    const int64_t tiles = (k.T + k.slots) * ((k.K + kWide - 1) / kWide) * ((k.N + kWide - 1) / kWide);
    k.window = xcd_window(tiles);
    const int64_t grid = xcd_grid(tiles, k.window);
    if (grid >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many tiles");
    hipLaunchKernelGGL((typed_wgrad_wide_kernel<T>), flat_grid(grid), dim3(256), 0, s, k);
    return RGNN_OK;
}

// The tile of a call with this plan; el: bytes of an element, any: rows on any address.
struct WgradTile { int bk, bn; };
WgradTile choose_tile(const WgradK &k, const WgradPlan &p, int el, bool any)
{
    // The wide tile takes rows as they are, at 32-bit offsets in a step.  Where it is not to be had, 128 x 128 walks the
    // pieces that the plan made for it (bf16, rows as they are and gathered, with the join: 8192 rows of 16 types, 2048 x 1536 97
    // and 192 us; 8192 rows of one type, 4096 x 4096 332 and 804; 4099 rows of 16 types, 1000 x 1040 41 and 62).
    if (el == 2 && p.bk == 256 && (any || k.gather || k.dy_gather || std::max(k.ldx, k.lddy) * kWide >= (int64_t(1) << 32))) return {128, 128};
    return {p.bk, p.bn};
}

template <class T, bool ANY>
rgnn_status launch_shape(const WgradK &k, const WgradPlan &p, hipStream_t s)
{
    if constexpr (sizeof(typename T::elem) == 4) {       // wgrad_plan
        return launch_tile<T, 64, 64, 2, 2, ANY>(k, s);
    } else {
        const WgradTile t = choose_tile(k, p, 2, ANY);
        if constexpr (!ANY)
            if (t.bk == 256) return launch_wide<T>(k, s);
        if (t.bk == 128 && t.bn == 128) return launch_tile<T, 128, 128, 2, 2, ANY>(k, s);
        if (t.bk == 128) return launch_tile<T, 128, 64, 2, 2, ANY>(k, s);
        if (t.bn == 128) return launch_tile<T, 64, 128, 2, 2, ANY>(k, s);
        return launch_tile<T, 64, 64, 2, 2, ANY>(k, s);
    }
}

template <class T>
rgnn_status launch_type(const WgradK &k, const WgradPlan &p, bool whole, hipStream_t s)
{
    return whole ? launch_shape<T, false>(k, p, s) : launch_shape<T, true>(k, p, s);
}

}  // namespace

WgradPlan wgrad_plan(int dtype, int64_t M, int32_t T, int32_t K, int32_t N)
{
    WgradPlan p;
    p.bk = K <= 64 ? 64 : 128;
    p.bn = N <= 64 ? 64 : 128;
    auto tiles = [&](int64_t b) { return (K + b - 1) / b * ((N + b - 1) / b); };
    const int64_t small = tiles(64);
    // 64 x 64 where little work is to be spread over the chip, and for fp32, bound by matrix cores that
    // take as long for a tile's empty part (10 007 rows of 7 types, 100 x 77: 16 us, 128 x 128 25; bf16, 292
    // rows, 1561 x 333: 17, 19; 20 000 rows, 512 x 512: 47, 39); the widest where its tiles alone fill the chip
    if (dtype == RGNN_F32 || (M * small <= 1 << 19 && T * small <= 1024)) p.bk = p.bn = 64;
    else if (K > 128 && N > 128 && tiles(256) * T >= 256) p.bk = p.bn = 256;
    const int64_t own = (int64_t)((K + p.bk - 1) / p.bk) * ((N + p.bn - 1) / p.bn);
    // pieces: enough workgroups over all tiles, and rows enough to pay for a piece's sums,
    // which are written and read back in fp32
    const int64_t want = dtype == RGNN_F32 ? 1024 : 512, least = p.bk == 256 ? 4096 : 128;
    p.chunk = std::max<int64_t>(least, (M * own + want - 1) / want);
    p.chunk = (p.chunk + 63) / 64 * 64;
    // A type is not cut where its walk takes less than the join: 256 rows (fp32, 1212 rows of 3 types, 40 x
    // 104: 12 us, up to 512 whole 18), or 1024 where the tiles fill the chip as they are (3916 rows of 5 types, 368 x
    // 712, bf16: 19 us, at 512 27).
    const int64_t least_whole = T * own >= 256 ? 1024 : 256;
    p.whole = std::max(p.chunk, least_whole);
    // rows / chunk + 1 of at most M / whole types; written so that it never falls as M grows
    p.slots = std::min(M / least, want / own) + std::min(M / least_whole, want / own);
    return p;
}

size_t wgrad_workspace(int dtype, int64_t M, int32_t T, int32_t K, int32_t N)
{
    return (size_t)wgrad_plan(dtype, M, T, K, N).slots * K * N * sizeof(float);
}

namespace {

bool whole_rows(const WgradArgs &a)
{
    const int el = dtype_bytes(a.dtype);
    return (uintptr_t)a.X % 16 == 0 && (uintptr_t)a.dY % 16 == 0 && a.ldx * el % 16 == 0 && a.lddy * el % 16 == 0 &&
           (int64_t)a.K * el % 16 == 0 && (int64_t)a.N * el % 16 == 0;
}

WgradK wgrad_args(const WgradArgs &a, const WgradPlan &plan)
{
    const int el = dtype_bytes(a.dtype);
    WgradK k{};
    k.X = (const char *)a.X; k.x_rows = a.x_rows; k.ldx = a.ldx * el; k.gather = a.gather;
    k.dY = (const char *)a.dY; k.dy_rows = a.dy_rows; k.lddy = a.lddy * el; k.dy_gather = a.dy_gather;
    k.x_end = k.X + ((a.x_rows - 1) * a.ldx + a.K) * el;
    k.dy_end = k.dY + ((a.dy_rows - 1) * a.lddy + a.N) * el;
    k.ptr = a.type_ptr; k.T = a.T; k.M = a.M; k.K = a.K; k.N = a.N;
    k.dW = a.dW; k.f32 = a.dw_dtype == RGNN_F32;
    k.cut = Cut{plan.whole, plan.chunk}; k.slots = plan.slots; k.partial = (float *)a.ws;
    return k;
}

}  // namespace

rgnn_tile_t typed_wgrad_tile(const WgradArgs &a)
{
    const WgradPlan plan = wgrad_plan(a.dtype, a.M, a.T, a.K, a.N);
    const bool any = !whole_rows(a);
    const WgradTile t = choose_tile(wgrad_args(a, plan), plan, dtype_bytes(a.dtype), any);
    return {t.bk, t.bn, t.bk == 256 ? 4 : 2, any};
}

rgnn_status launch_typed_wgrad(const WgradArgs &a, hipStream_t s)
{
    const WgradPlan plan = wgrad_plan(a.dtype, a.M, a.T, a.K, a.N);
    const bool whole = whole_rows(a);
    const WgradK k = wgrad_args(a, plan);
    rgnn_status st;
    {
        LaunchScope ls("typed_wgrad", s);
        st = a.dtype == RGNN_F32 ? launch_type<F32>(k, plan, whole, s)
             : a.dtype == RGNN_BF16 ? launch_type<BF16>(k, plan, whole, s) : launch_type<F16>(k, plan, whole, s);
    }
    if (st != RGNN_OK) return st;
    if (plan.slots > 0) {
        if (a.dtype == RGNN_F32) launch_join<float>(a, plan, s);
        else if (a.dtype == RGNN_BF16) launch_join<__bf16>(a, plan, s);
        else launch_join<_Float16>(a, plan, s);
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "typed_wgrad launch");
}

}  // namespace rgnn
