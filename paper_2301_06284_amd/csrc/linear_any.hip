// linear_any.hip -- the typed linear and its weight gradient for sizes, strides and
// addresses that fill no vector of 16 bytes.
#include <algorithm>

#include "linear_ops.h"

namespace rgnn {

namespace {

// ---------------------------------------------------------------- any sizes
//
// The form without any demand on sizes, strides and alignment: 64 x 64 outputs a
// workgroup of four waves (32 x 32 each), both operands taken element by element into
// LDS rows of 64 bytes of k, zero outside the matrix, and multiplied by the matrix
// cores from there.  Bound by the element loads.

constexpr int kAny = 64;         // outputs of a tile, each way
constexpr int kAnyRow = 80;      // bytes of an LDS row: 64 of k and 16 against bank conflicts

enum AnyOp { kForward, kTransposed, kWgrad };

struct AnyArgs {
    const void *A, *B;           // X (or X of the weight gradient); W or dY
    int64_t a_rows, lda, b_rows, ldb;
    const int32_t *a_index, *b_index;   // gather of X; of dY (weight gradient)
    const int64_t *ptr;
    int T;
    int64_t M;
    int K, N;                    // of the weights as the call names them
    void *out;                   // Y or dW
    int64_t out_rows, ldo;
    const int32_t *scatter;
    int out_f32;
    int64_t chunk;               // weight gradient: rows of a piece
    float *partial;              // and the sums of types with several pieces [slots, K, N]
    int64_t slots;
};

template <class E>
__device__ __forceinline__ void store_out(void *out, int64_t at, float v, int f32)
{
    if (f32) ((float *)out)[at] = v;
    else ((E *)out)[at] = (E)v;
}

template <class T, int OP>
__global__ __launch_bounds__(256, 2) void linear_any_kernel(AnyArgs a)
{
    typedef typename T::elem E;
    constexpr int KE = 64 / sizeof(E);               // k of a step
    constexpr int RE = kAnyRow / sizeof(E);
    __shared__ __attribute__((aligned(16))) E sa[kAny * RE], sb[kAny * RE];
    const E *A = (const E *)a.A, *B = (const E *)a.B;
    const int ni = OP == kWgrad ? (a.K + kAny - 1) / kAny : 1;
    const int nj = (a.N + kAny - 1) / kAny;
    Piece p;
    const int64_t chunk = a.chunk;
    const int64_t per = (int64_t)ni * nj;
    const bool any = OP == kWgrad
        ? find_piece(a.ptr, a.T, a.M, blockIdx.x,
                     [=](int64_t c) { return (c <= chunk ? 1 : (c + chunk - 1) / chunk) * per; },
                     [=](int64_t c) { return c <= chunk ? 0 : (c + chunk - 1) / chunk; }, p)
        : find_piece(a.ptr, a.T, a.M, blockIdx.x,
                     [=](int64_t c) { return (c + kAny - 1) / kAny * nj; }, NoWeight(), p);
    if (!any) return;
    const int64_t part = p.index / per;              // row tile, or piece of the contraction
    const int64_t rest = p.index % per;
    const int j0 = (int)(rest % nj) * kAny;
    const int64_t i0 = OP == kWgrad ? rest / nj * kAny : p.begin + part * kAny;
    const int64_t i1 = OP == kWgrad ? a.K : p.end;
    const int64_t k0 = OP == kWgrad ? p.begin + part * chunk : 0;
    const int64_t k1 = OP == kWgrad ? (k0 + chunk < p.end ? k0 + chunk : p.end) : a.K;
    const E *W = B + (OP == kWgrad ? 0 : (int64_t)p.type * a.K * a.N);

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    f32x4 acc[2][2] = {};
    for (int64_t ks = k0; ks < k1; ks += KE) {
        // A: row i, k (forward: k along the lanes; weight gradient: i)
        for (int x = tid; x < kAny * KE; x += 256) {
            const int i = OP == kWgrad ? x % kAny : x / KE, k = OP == kWgrad ? x / kAny : x % KE;
            E v = (E)0.0f;
            if (i0 + i < i1 && ks + k < k1) {
                int64_t row = OP == kWgrad ? ks + k : i0 + i;
                const int64_t col = OP == kWgrad ? i0 + i : ks + k;
                if (a.a_index) row = a.a_index[row];
                if (row >= 0 && row < a.a_rows) v = A[row * a.lda + col];
            }
            sa[i * RE + k] = v;
        }
        for (int x = tid; x < kAny * KE; x += 256) {
            const int j = OP == kTransposed ? x / KE : x % kAny, k = OP == kTransposed ? x % KE : x / kAny;
            E v = (E)0.0f;
            if (j0 + j < a.N && ks + k < k1) {
                if (OP == kForward) v = W[(ks + k) * a.N + j0 + j];
                else if (OP == kTransposed) v = W[(int64_t)(j0 + j) * a.K + ks + k];
                else {
                    int64_t row = ks + k;
                    if (a.b_index) row = a.b_index[row];
                    if (row >= 0 && row < a.b_rows) v = B[row * a.ldb + j0 + j];
                }
            }
            sb[j * RE + k] = v;
        }
        __syncthreads();
        const int r = lane & 15, c = lane >> 4;
        i32x4 fa[2], fb[2];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            fa[f] = *(const i32x4 *)((const char *)sa + ((wave >> 1) * 32 + f * 16 + r) * kAnyRow + c * 16);
            fb[f] = *(const i32x4 *)((const char *)sb + ((wave & 1) * 32 + f * 16 + r) * kAnyRow + c * 16);
        }
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) acc[f][h] = mma16<T>(fb[h], fa[f], acc[f][h]);
        __syncthreads();
    }
    const bool split = OP == kWgrad && p.end - p.begin > chunk;
    const int64_t slot = p.before + part;
    if (split && slot >= a.slots) return;            // only where the offsets are not monotone
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        const int64_t i = i0 + (wave >> 1) * 32 + f * 16 + (lane & 15);
        if (i >= i1) continue;
        int64_t row = i;
        if (OP != kWgrad) {
            if (a.scatter) row = a.scatter[i];
            if (row < 0 || row >= a.out_rows) continue;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = j0 + (wave & 1) * 32 + h * 16 + (lane >> 4) * 4 + q;
                if (j >= a.N) continue;
                if (OP != kWgrad) store_out<E>(a.out, row * a.ldo + j, acc[f][h][q], a.out_f32);
                else if (split) a.partial[(slot * a.K + i) * a.N + j] = acc[f][h][q];
                else store_out<E>(a.out, ((int64_t)p.type * a.K + i) * a.N + j, acc[f][h][q], a.out_f32);
            }
    }
}

template <int OP>
bool launch_any(int dtype, const AnyArgs &k, int64_t grid, hipStream_t s)
{
    switch (dtype) {
    case RGNN_F32: hipLaunchKernelGGL((linear_any_kernel<F32, OP>), dim3((uint32_t)grid), dim3(256), 0, s, k); return true;
    case RGNN_BF16: hipLaunchKernelGGL((linear_any_kernel<BF16, OP>), dim3((uint32_t)grid), dim3(256), 0, s, k); return true;
    case RGNN_F16: hipLaunchKernelGGL((linear_any_kernel<F16, OP>), dim3((uint32_t)grid), dim3(256), 0, s, k); return true;
    }
    return false;
}

}  // namespace

rgnn_status launch_linear_any(const LinearArgs &a, hipStream_t s)
{
    AnyArgs k{};
    k.A = a.X; k.a_rows = a.x_rows; k.lda = a.ldx; k.a_index = a.gather;
    k.B = a.W;
    k.ptr = a.type_ptr; k.T = a.T; k.M = a.M; k.K = a.K; k.N = a.N;
    k.out = a.Y; k.out_rows = a.y_rows; k.ldo = a.ldy; k.scatter = a.scatter;
    k.out_f32 = a.y_dtype == RGNN_F32;
    const int64_t grid = row_tiles_bound(a.M, a.T, kAny) * ((a.N + kAny - 1) / kAny);
    if (grid >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many tiles");
    {
        LaunchScope ls("typed_linear_any", s);
        if (!(a.trans_w ? launch_any<kTransposed>(a.dtype, k, grid, s) : launch_any<kForward>(a.dtype, k, grid, s)))
            return fail(RGNN_EUNSUPPORTED, "typed linear: unsupported type");
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "typed_linear launch");
}

rgnn_status launch_wgrad_any(const WgradArgs &a, const WgradPlan &plan, hipStream_t s)
{
    AnyArgs k{};
    k.A = a.X; k.a_rows = a.x_rows; k.lda = a.ldx; k.a_index = a.gather;
    k.B = a.dY; k.b_rows = a.dy_rows; k.ldb = a.lddy; k.b_index = a.dy_gather;
    k.ptr = a.type_ptr; k.T = a.T; k.M = a.M; k.K = a.K; k.N = a.N;
    k.out = a.dW; k.out_f32 = a.dw_dtype == RGNN_F32;
    k.chunk = plan.chunk; k.partial = (float *)a.ws; k.slots = plan.slots;
    const int64_t tiles = (int64_t)((a.K + kAny - 1) / kAny) * ((a.N + kAny - 1) / kAny);
    const int64_t grid = (a.T + plan.slots) * tiles;
    if (grid >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many tiles");
    {
        LaunchScope ls("typed_wgrad_any", s);
        if (!launch_any<kWgrad>(a.dtype, k, grid, s)) return fail(RGNN_EUNSUPPORTED, "weight gradient: unsupported type");
    }
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "typed_wgrad launch");
}

}  // namespace rgnn
