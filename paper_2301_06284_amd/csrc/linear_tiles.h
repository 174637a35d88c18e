// linear_tiles.h -- device code that the tiled kernels of the typed linear and of its
// weight gradient share: loads into LDS, the LDS layouts, the order of tiles, writing.
#pragma once

#include "linear_ops.h"

namespace rgnn {

static __device__ const i32x4 kZeros = {0, 0, 0, 0};

typedef const __attribute__((address_space(1))) uint32_t *global_ptr;
typedef __attribute__((address_space(3))) uint32_t *lds_ptr;

// 16 bytes of every lane's address to LDS, lane after lane from `lds` on
__device__ __forceinline__ void load_lds(const char *from, char *lds)
{
    __builtin_amdgcn_global_load_lds((global_ptr)from, (lds_ptr)lds, 16, 0, 0);
}

// Every wave's loads into LDS, but for its UNDER youngest, have arrived, and every wave has
// read what it wanted of the step before.  (A __syncthreads() would wait for all loads.)  The
// empty asm statements keep the compiler from moving reads and loads across.
template <int UNDER>
__device__ __forceinline__ void step_barrier()
{
    static_assert(UNDER < 64, "vmcnt has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (UNDER & 15) | (UNDER >> 4) << 14);   // vmcnt(UNDER) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 *lds_i16x4;
__device__ __forceinline__ uint64_t read_turned(const char *lds)
{
    return __builtin_bit_cast(uint64_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4)lds));
}

// How the 32-byte units (16-bit) or 64-byte units (fp32) of row k are permuted.
template <class T, int BN>
__device__ __forceinline__ int unit_turn(int k)
{
    if (sizeof(typename T::elem) == 4) return (k >> 2) & 3;
    return BN >= 128 ? (k & 3) | ((k >> 1) & 4) : ((k >> 1) & 1) | ((k >> 2) & 2);
}

// Order of a type's tiles: groups of 8 row tiles, in a group all row tiles of one column
// tile after another, so that the tiles at work together share rows and weights in L2.
__device__ __forceinline__ void tile_place(int q, int mt, int nt, int &m, int &n)
{
    const int group = q / (8 * nt), rest = q - group * 8 * nt;
    const int gm = min(8, mt - group * 8);
    n = rest / gm;
    m = group * 8 + rest - n * gm;
}

// Four outputs side by side, or the first `n` of them.
template <class O>
__device__ __forceinline__ void write4(O *y, f32x4 v, bool whole, int n)
{
    O o[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] = (O)v[q];
    if (whole) {
        if constexpr (sizeof(O) == 2) *(uint2 *)y = *(const uint2 *)o;
        else *(i32x4 *)y = *(const i32x4 *)o;
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < n) y[q] = o[q];
    }
}

// XCD windows: up to 32 tiles for each of the 8 XCDs, an eighth of the work at most.
inline int xcd_window(int64_t tiles)
{
    int window = 32;
    while (window > 1 && (int64_t)window * 8 * 4 > tiles) window /= 2;
    return window;
}
inline int64_t xcd_grid(int64_t tiles, int window) { return (tiles + window * 8 - 1) / (window * 8) * (window * 8); }

// The tile of a workgroup: each XCD, which takes every eighth workgroup, gets neighbours.
__device__ __forceinline__ int xcd_tile(int window)
{
    const uint32_t in = blockIdx.x & (uint32_t)(window * 8 - 1);   // a power of two
    return (int)(blockIdx.x - in + (in & 7) * window + (in >> 3));
}

}  // namespace rgnn
