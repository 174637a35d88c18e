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

// Four outputs side by side, or the first `n` of them, to any address of an element.
template <class O>
__device__ __forceinline__ void write4(O *y, f32x4 v, int n)
{
    O o[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] = (O)v[q];
    if (n >= 4) __builtin_memcpy(y, o, sizeof(o));
    else
#pragma unroll
        for (int q = 0; q < 3; ++q)
            if (q < n) y[q] = o[q];
}

// Eight 16-bit outputs side by side, or the first `n` of them (none for n <= 0), to any address.
template <class O>
__device__ __forceinline__ void write8(O *y, i32x4 v, int n)
{
    if (n >= 8) __builtin_memcpy(y, &v, 16);
    else {
        O o[8];
        __builtin_memcpy(o, &v, 16);
#pragma unroll
        for (int q = 0; q < 7; ++q)
            if (q < n) y[q] = o[q];
    }
}

// Writes a wave's outputs in 16 bits through LDS (FM * FN * 512 bytes of its own), so that rows
// go out in pieces as wide as the wave's columns: from the accumulators a store would take 32 bytes each of
// 16 rows.  `y` points at the wave's first column, of which `cols` are the matrix's.  Chunk c of row r
// lies at c ^ (r >> 1 & 7) (FN = 4) or c ^ (r >> 2 & 3) (FN = 2): no bank conflicts.
// to[r]: where row r goes, -1 nowhere; below -1: zeros to row -2 - to[r].
template <class O, int FM, int FN>
__device__ __forceinline__ void write_rows(char *lds, const f32x4 (&acc)[FM][FN], O *y, int64_t ldy, int cols, int lane,
                                           const int *to)
{
    static_assert(FN == 2 || FN == 4, "pieces of 64 or 128 bytes");
    constexpr int CH = FN * 2;                      // chunks of a row
    auto turn = [](int r) { return FN == 4 ? r >> 1 & 7 : r >> 2 & 3; };
    const int r16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int m = 0; m < FM; ++m)
#pragma unroll
        for (int f = 0; f < FN; ++f) {
            O o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = (O)acc[m][f][q];
            *(uint2 *)(lds + (m * 16 + r16) * (CH * 16) + ((f * 2 + (g >> 1)) ^ turn(r16)) * 16 + (g & 1) * 8) = *(const uint2 *)o;
        }
    // a wave's LDS instructions stay in order: its reads see its writes
    const int c = lane % CH, left = cols - c * 8;   // this lane's columns
#pragma unroll
    for (int t = 0; t < FM * FN / 2; ++t) {
        const int r = t * (64 / CH) + lane / CH;
        i32x4 v = *(const i32x4 *)(lds + r * (CH * 16) + (c ^ turn(r)) * 16);
        int row = to[r];
        if (row < -1) { row = -2 - row; v = i32x4{0, 0, 0, 0}; }
        if (row >= 0) write8(y + row * ldy + c * 8, v, left);
    }
}

// 16 bytes from any address of an element; by elements, zero behind `end`, where they would
// reach behind it.
template <class E>
__device__ __forceinline__ i32x4 load_any(const char *p, const char *end)
{
    i32x4 v = {0, 0, 0, 0};
    if (p + 16 <= end) {
        __builtin_memcpy(&v, p, 16);
    } else {
        E e[16 / sizeof(E)];
#pragma unroll
        for (int i = 0; i < (int)(16 / sizeof(E)); ++i)
            e[i] = p + (i + 1) * sizeof(E) <= end ? ((const E *)p)[i] : (E)0.0f;
        __builtin_memcpy(&v, e, 16);
    }
    return v;
}

// The first n bytes of v, the others zero.
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int n)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = n - i * 4;
        v[i] = left >= 4 ? v[i] : left <= 0 ? 0 : v[i] & ((1 << left * 8) - 1);
    }
    return v;
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
    const uint32_t block = flat_block(), in = block & (uint32_t)(window * 8 - 1);   // a power of two
    return (int)(block - in + (in & 7) * window + (in >> 3));
}

}  // namespace rgnn
