// linear_ops.h -- what the typed linear's kernels share: element types and their
// matrix instructions, the search for a workgroup's tile in offsets that lie on the
// device, and the launchers' arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "rgnn_internal.h"

namespace rgnn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- arguments

struct LinearArgs {
    int dtype = 0;                       // rgnn_dtype of X and W (fp8: RGNN_F8_E4M3)
    int y_dtype = 0;
    const void *X = nullptr;   int64_t x_rows = 0, ldx = 0;
    const int32_t *gather = nullptr;
    const int64_t *type_ptr = nullptr;   // device [T+1]
    int32_t T = 0;
    int64_t M = 0;
    const void *W = nullptr;
    int32_t K = 0, N = 0;
    int trans_w = 0;                     // W stored [T, N, K]
    void *Y = nullptr;         int64_t y_rows = 0, ldy = 0;
    const int32_t *scatter = nullptr;
    // fp8: scale bytes of X [x_rows, ks] and of W [T, ceil(N/128), ks]
    const uint8_t *x_scale = nullptr, *w_scale = nullptr;
};

struct WgradArgs {
    int dtype = 0, dw_dtype = 0;
    const void *X = nullptr;   int64_t x_rows = 0, ldx = 0;
    const int32_t *gather = nullptr;     // rows of X
    const void *dY = nullptr;  int64_t dy_rows = 0, lddy = 0;
    const int32_t *dy_gather = nullptr;  // rows of dY (the forward's scatter)
    const int64_t *type_ptr = nullptr;
    int32_t T = 0;
    int64_t M = 0;
    int32_t K = 0, N = 0;
    void *dW = nullptr;
    void *ws = nullptr;
};

// How the weight gradient's contraction is cut: types with more rows than `whole` into pieces of
// `chunk` rows, and how many pieces those can be (their sums go through the workspace).
struct WgradPlan {
    int bk = 0, bn = 0;          // the tile
    int64_t whole = 0, chunk = 0, slots = 0;
};
WgradPlan wgrad_plan(int dtype, int64_t M, int32_t T, int32_t K, int32_t N);
size_t wgrad_workspace(int dtype, int64_t M, int32_t T, int32_t K, int32_t N);
rgnn_status launch_typed_linear(const LinearArgs &a, hipStream_t s);
rgnn_status launch_typed_wgrad(const WgradArgs &a, hipStream_t s);
rgnn_tile_t typed_linear_tile(const LinearArgs &a);     // what the launchers take, for fp8 too
rgnn_tile_t typed_wgrad_tile(const WgradArgs &a);

rgnn_status launch_typed_fp8(const LinearArgs &a, hipStream_t s);
rgnn_status launch_fp8_rows(int dtype, const void *X, int64_t rows, int64_t ldx, int K, void *codes, uint8_t *scales,
                            hipStream_t s);
rgnn_status launch_fp8_weights(int dtype, const void *W, int T, int K, int N, void *codes, uint8_t *scales, hipStream_t s);
rgnn_status launch_adamw(const rgnn_adamw_tensor_t *t, int32_t count, const rgnn_adamw_t &h, int64_t step,
                         const int64_t *step_dev, const float *grad_scale, hipStream_t s);

// Width of the codes of K elements, and bytes of their scales (whole words).
constexpr int32_t fp8_width(int32_t K) { return (K + 127) / 128 * 128; }
constexpr int32_t fp8_scales(int32_t K) { return (K + 511) / 512 * 4; }

constexpr int dtype_bytes(int d) { return d == RGNN_F32 ? 4 : d == RGNN_F8_E4M3 ? 1 : 2; }

// Row tiles of `rows` rows that M rows of T types can make, at most: every type that
// has rows can leave one tile partly filled.
inline int64_t row_tiles_bound(int64_t M, int64_t T, int64_t rows)
{
    const int64_t nz = M < T ? M : T;
    return (M + nz * (rows - 1)) / rows;
}

#ifdef __HIPCC__

// A launch holds fewer than 2^32 threads along x: `groups` workgroups (fewer than 2^31) in rows of 2^22.
inline dim3 flat_grid(int64_t groups)
{
    constexpr int64_t row = int64_t(1) << 22;
    return groups <= row ? dim3((uint32_t)groups) : dim3((uint32_t)row, (uint32_t)((groups + row - 1) / row));
}
__device__ __forceinline__ uint32_t flat_block() { return blockIdx.y * gridDim.x + blockIdx.x; }

// ---------------------------------------------------------------- elements

struct F32 { typedef float elem; };
struct BF16 { typedef __bf16 elem; };
struct F16 { typedef _Float16 elem; };

// D[n][m] += sum_k a[n][k] b[m][k] over 16 bytes of k a lane: lane l holds row l % 16
// of both, 16-byte chunk l / 16 of the step's k.  The order of k within a step is the
// same for both operands, so any one will do: fp32 takes the chunk's element i of the
// four lane groups in instruction i.  The result's lane l holds m = l % 16 and the
// four n = 4 (l / 16) + i.
template <class T>
__device__ __forceinline__ f32x4 mma16(i32x4 a, i32x4 b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 mma16<BF16>(i32x4 a, i32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 mma16<F16>(i32x4 a, i32x4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 mma16<F32>(i32x4 a, i32x4 b, f32x4 c)
{
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
    return c;
}

// ---------------------------------------------------------------- tiles

struct Piece {          // a workgroup's share: number `index` of type `type`'s pieces
    int type;
    int64_t begin, end;   // the type's rows, inside [0, M)
    int index;            // which of the type's pieces
    int before;           // what `weight` counted in the types before it
};

// Sum over the lanes up to this one, on DPP (no LDS): within rows of 16, then across rows.
__device__ __forceinline__ int wave_prefix_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);   // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);   // row_shr:2
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);   // row_shr:4
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);   // row_shr:8
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);   // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);   // row_bcast:31 into rows 2 and 3
    return x;
}

// The same for the largest; x >= 0.
__device__ __forceinline__ int wave_prefix_max(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));
    return max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));
}

struct NoWeight {
    __device__ __forceinline__ int operator()(int64_t) const { return 0; }
};

// The type that owns piece number `want`, where a type with c rows makes count(c) pieces (fewer
// than 2^31 over all types: the host checks the grid).  Every wave of a workgroup searches
// alike, 256 types a turn: one load of the offsets and prefix sums over the lanes, no LDS and no
// barrier.  weight(c) is a second count summed over the types before the owner.  False where
// there are fewer pieces.
//
// The host has not seen the offsets: they are kept inside [0, M), and one below an earlier one
// counts as that (a running maximum), so that the types' rows never overlap and the counts
// over all types stay within what the host sized grid and workspace for.
template <class Count, class Weight>
__device__ __forceinline__ bool find_piece(const int64_t *__restrict__ ptr, int T, int64_t M, int want,
                                           Count count, Weight weight, Piece &out)
{
    constexpr bool WEIGHT = !std::is_same<Weight, NoWeight>::value;
    const int lane = threadIdx.x & 63, most = (int)M;
    int before = 0, wbefore = 0, top = 0;
    for (int t0 = 0; t0 < T; t0 += 256) {
        int at[5], c[4], w[4], cs = 0, ws = 0;
        int64_t raw[5];      // loads that depend on nothing, all at once
#pragma unroll
        for (int i = 0; i < 5; ++i) raw[i] = ptr[min(t0 + lane * 4 + i, T)];
#pragma unroll
        for (int i = 0; i < 5; ++i) at[i] = raw[i] < 0 ? 0 : raw[i] > M ? most : (int)raw[i];
        at[0] = max(at[0], top);
#pragma unroll
        for (int i = 1; i < 5; ++i) at[i] = max(at[i], at[i - 1]);
        const int upto = wave_prefix_max(at[4]);
        const int earlier = __builtin_amdgcn_update_dpp(0, upto, 0x138, 0xF, 0xF, false);   // wave_shr:1
#pragma unroll
        for (int i = 0; i < 5; ++i) at[i] = max(at[i], earlier);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool own = t0 + lane * 4 + i < T;
            c[i] = own ? (int)count(at[i + 1] - at[i]) : 0;
            w[i] = own ? (int)weight(at[i + 1] - at[i]) : 0;
            cs += c[i];
            ws += w[i];
        }
        const int ci = wave_prefix_sum(cs), wi = WEIGHT ? wave_prefix_sum(ws) : 0;
        const int total = __builtin_amdgcn_readlane(ci, 63);
        if (want < before + total) {
            const uint64_t over = __ballot(before + ci > want);
            const int owner = __builtin_ctzll(over);
            int pat = before + ci - cs, wat = wbefore + wi - ws;   // before this lane's first type
            int k = 0;
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (k == i && pat + c[i] <= want) { pat += c[i]; wat += w[i]; k = i + 1; }
            const int bb = k == 0 ? at[0] : k == 1 ? at[1] : k == 2 ? at[2] : at[3];
            const int ee = k == 0 ? at[1] : k == 1 ? at[2] : k == 2 ? at[3] : at[4];
            out.type = t0 + owner * 4 + __builtin_amdgcn_readlane(k, owner);
            out.begin = __builtin_amdgcn_readlane(bb, owner);
            out.end = __builtin_amdgcn_readlane(ee, owner);
            out.index = want - __builtin_amdgcn_readlane(pat, owner);
            out.before = WEIGHT ? __builtin_amdgcn_readlane(wat, owner) : 0;
            return true;
        }
        before += total;
        if (WEIGHT) wbefore += __builtin_amdgcn_readlane(wi, 63);
        top = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

#endif  // __HIPCC__

}  // namespace rgnn
