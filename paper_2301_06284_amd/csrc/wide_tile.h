// wide_tile.h -- the 256 x 256 tile that the typed linear and its weight gradient share:
// four waves, one for each SIMD of a CU, 128 x 128 outputs each.
//
// At this size the matrix cores ask least of LDS: a wave reads 256 rows of a step for 128 x 128
// products, so that the four waves' reads and the step's own arrival take 768 LDS cycles beside 1024 of
// the matrix cores (eight waves of 128 x 64: 1024 beside 1024, which measured half of them idle).
// With a single wave on a SIMD nothing else hides a wait, so the walk over k is laid out
// in advance: steps of 64 bytes of k in four LDS stages, the fragments of the next step read
// while this step's are multiplied, three more steps on their way from memory.
//
// Measured, calls queued one after another: 4096 columns, bf16, 16 384 rows, k of 2048 242 us (1.14 PFLOP/s), of 8192
// 1.36 PFLOP/s; 8 bits, 8192 rows, k of 4096 1.93, of 8192 2.2.  64 steps take 83 000 cycles, 65 500 of them the matrix cores'; a
// tile's outputs 13 000 to 16 000 more, as all CUs write at once.
#pragma once

#include "linear_tiles.h"

namespace rgnn {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kWide = 256, kWideKB = 64;             // tile, bytes of k of a step
constexpr int kWideStage = kWide * kWideKB;          // bytes of one operand's stage
constexpr int kWideLoads = kWideStage / 1024 / 4;    // loads of a wave and operand each step

// D[n][m] += a[n][k] b[m][k] over 32 rows each: lane l holds row l % 32, chunks l / 32 and
// l / 32 + 2 of the 64 bytes of k (16-bit: an instruction each; 8-bit: one of both).  The
// result's lane holds m = l % 32 and n = 8 (i / 4) + 4 (l / 32) + i % 4, i = 0 .. 15.
template <class T>
__device__ __forceinline__ f32x16 mma32(i32x4 a, i32x4 b, f32x16 c);
template <>
__device__ __forceinline__ f32x16 mma32<BF16>(i32x4 a, i32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x16 mma32<F16>(i32x4 a, i32x4 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Chunk q of a fragment.
__device__ __forceinline__ i32x4 chunk_of(i32x8 v, int q)
{
    return q ? __builtin_shufflevector(v, v, 4, 5, 6, 7) : __builtin_shufflevector(v, v, 0, 1, 2, 3);
}

// LDS rows of 64 bytes of k: chunk c of row r lies at c ^ (r >> 3 & 3).  A 16-byte read takes lanes
// 0-3, 12-15, 20-23, 24-27 of 32 together and the others together: with this turn their chunks
// lie in different banks (no conflicts by the counters).
__device__ __forceinline__ int wide_turn_k(int row) { return row >> 3 & 3; }
// LDS rows of 256 16-bit values for each k: unit u of 32 bytes of row k lies at u ^ (k & 3) << 1.
__device__ __forceinline__ int wide_turn_n(int k) { return (k & 3) << 1; }

// One operand's fragment of 32 rows: chunk q of this lane.  COLS: kept as rows of n.
template <bool COLS>
struct WideFragments {
    int at;       // this lane's place in a stage, of fragment 0
    __device__ __forceinline__ void init(int first_row, int lane)   // the wave's first row (COLS: column)
    {
        if (COLS) {
            const int k = (lane >> 5) * 8 + (lane >> 2 & 3);
            at = k * 512 + ((first_row / 16 + (lane >> 4 & 1)) ^ wide_turn_n(k)) * 32 + (lane & 3) * 8;
        } else {
            const int row = first_row + (lane & 31);
            at = row * 64 + ((lane >> 5) ^ wide_turn_k(row)) * 16;
        }
    }
    __device__ __forceinline__ i32x4 read(const char *stage, int f, int q) const
    {
        if (COLS) {     // f moves the unit by 2 f, above the turn's bits and among them: an exclusive or
            const char *p = stage + (at ^ f * 64) + q * 16 * 512;
            const uint64_t x = read_turned(p), y = read_turned(p + 4 * 512);
            return i32x4{(int)x, (int)(x >> 32), (int)y, (int)(y >> 32)};
        }
        return *(const i32x4 *)(stage + (at ^ q * 32) + f * 32 * 64);
    }
};

// One operand's loads: a base that all lanes share and moves from step to step, and an offset
// for each of a lane's rows that does not; so a load costs one instruction and no address.
struct WideSide {
    const char *base;
    int64_t step;                    // bytes from one step to the next
    uint32_t off[kWideLoads];
    template <int L>
    __device__ __forceinline__ void load(char *stage, int wave)
    {
#pragma unroll
        for (int x = 0; x < L; ++x) load_lds(base + off[x], stage + (x * 4 + wave) * 1024);
    }
    // a step that the matrix does not fill: lanes outside read zeros
    template <int L, class Inside>
    __device__ __forceinline__ void load_edge(char *stage, int wave, Inside inside)
    {
#pragma unroll
        for (int x = 0; x < L; ++x) load_lds(inside(x) ? base + off[x] : (const char *)&kZeros, stage + (x * 4 + wave) * 1024);
    }
};

// The walk over `steps` steps, of which `whole` are filled by the matrix, rounded up to four (what
// lies behind is zero).  FMV of a wave's four row fragments are used.  load(stage a, stage b): a
// wave's LA + LB loads of the next step; edge(stage a, stage b, step): the same where the step may
// not be whole.  shift(step): what a type needs before it multiplies a step.
template <int FMV, bool ACOLS, bool BCOLS, int LOADS, class Load, class Edge, class Multiply, class Shift>
__device__ __forceinline__ void wide_walk(char *a0, char *b0, char *a1, char *b1, char *a2, char *b2, char *a3, char *b3,
                                          const WideFragments<ACOLS> &fa, const WideFragments<BCOLS> &fb, int steps, int whole,
                                          Load load, Edge edge, Multiply multiply, Shift shift, f32x16 (&acc)[4][4])
{
    struct Set { i32x8 a[FMV], b[4]; };      // both chunks side by side
    auto fetch = [&](Set &s, const char *a, const char *b) {
#pragma unroll
        for (int n = 0; n < 4; ++n) s.b[n] = __builtin_shufflevector(fb.read(b, n, 0), fb.read(b, n, 1), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int m = 0; m < FMV; ++m) s.a[m] = __builtin_shufflevector(fa.read(a, m, 0), fa.read(a, m, 1), 0, 1, 2, 3, 4, 5, 6, 7);
    };
    // A wave's instructions issue in order: a load into LDS that waits for its turn holds up the
    // products behind it.  So reads and loads go between the products, as evenly as they can.
    auto spread = [&]() {
        constexpr int READS = 2 * (FMV * (ACOLS ? 2 : 1) + 4 * (BCOLS ? 2 : 1)), PRODUCTS = FMV * 4 * 2;
        constexpr int G = LOADS, R = (READS + G - 3) / (G - 2), P = PRODUCTS / G;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            if (i < G - 2) __builtin_amdgcn_sched_group_barrier(0x100, R, 0);   // LDS reads, the last ones before the step's end
            __builtin_amdgcn_sched_group_barrier(0x008, P / 2, 0);  // products
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);      // a load
            __builtin_amdgcn_sched_group_barrier(0x008, P - P / 2, 0);
        }
    };
    Set x, y;
    edge(a0, b0, 0);
    edge(a1, b1, 1);
    edge(a2, b2, 2);
    edge(a3, b3, 3);
    step_barrier<3 * LOADS>();
    fetch(x, a0, b0);
    int step = 0;
    for (; step + 8 <= whole; step += 4) {
        step_barrier<2 * LOADS>();
        load(a0, b0);
        fetch(y, a1, b1);
        shift(step);
        multiply(x.a, x.b, acc);
        spread();
        step_barrier<2 * LOADS>();
        load(a1, b1);
        fetch(x, a2, b2);
        shift(step + 1);
        multiply(y.a, y.b, acc);
        spread();
        step_barrier<2 * LOADS>();
        load(a2, b2);
        fetch(y, a3, b3);
        shift(step + 2);
        multiply(x.a, x.b, acc);
        spread();
        step_barrier<2 * LOADS>();
        load(a3, b3);
        fetch(x, a0, b0);
        shift(step + 3);
        multiply(y.a, y.b, acc);
        spread();
    }
    for (; step + 4 < steps; step += 4) {
        step_barrier<2 * LOADS>();
        edge(a0, b0, step + 4);
        fetch(y, a1, b1);
        shift(step);
        multiply(x.a, x.b, acc);
        step_barrier<2 * LOADS>();
        edge(a1, b1, step + 5);
        fetch(x, a2, b2);
        shift(step + 1);
        multiply(y.a, y.b, acc);
        step_barrier<2 * LOADS>();
        edge(a2, b2, step + 6);
        fetch(y, a3, b3);
        shift(step + 2);
        multiply(x.a, x.b, acc);
        step_barrier<2 * LOADS>();
        edge(a3, b3, step + 7);
        fetch(x, a0, b0);
        shift(step + 3);
        multiply(y.a, y.b, acc);
    }
    step_barrier<2 * LOADS>();
    fetch(y, a1, b1);
    shift(step);
    multiply(x.a, x.b, acc);
    step_barrier<LOADS>();
    fetch(x, a2, b2);
    shift(step + 1);
    multiply(y.a, y.b, acc);
    step_barrier<0>();
    fetch(y, a3, b3);
    shift(step + 2);
    multiply(x.a, x.b, acc);
    shift(step + 3);
    multiply(y.a, y.b, acc);
    step_barrier<0>();               // every wave has read the stages: they may be used again
}

// Writes a wave's FMV x 128 x 128 / 4 outputs in 16 bits through LDS (32 KB of its own), so that
// rows go out as whole pieces of 256 bytes: from the accumulators a store would take 16 bytes each
// of 32 rows.  `y` points at the wave's first column, of which `cols` are the matrix's.  Chunk c of row r lies at c ^ (r & 15), its halves exchanged where r & 16.
// to[r]: where row r of the wave goes, -1 nowhere; below -1: zeros to row -2 - to[r].
template <class O, int FMV>
__device__ __forceinline__ void wide_write(char *lds, const f32x16 (&acc)[4][4], O *y, int64_t ldy, int cols, int lane,
                                           const int *to)
{
    const int r32 = lane & 31, half = (lane >> 5) ^ (r32 >> 4);
#pragma unroll
    for (int m = 0; m < FMV; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                O o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (O)acc[m][n][q * 4 + i];
                *(uint2 *)(lds + (m * 32 + r32) * 256 + ((n * 4 + q) ^ (r32 & 15)) * 16 + half * 8) = *(const uint2 *)o;
            }
    // a wave's LDS instructions stay in order: its reads see its writes
#pragma unroll 4
    for (int t = 0; t < FMV * 8; ++t) {
        const int r = t * 4 + (lane >> 4), c = lane & 15;
        i32x4 v = *(const i32x4 *)(lds + r * 256 + (c ^ (r & 15)) * 16);
        if (r & 16) v = i32x4{v[2], v[3], v[0], v[1]};
        int row = to[r];
        if (row < -1) { row = -2 - row; v = i32x4{0, 0, 0, 0}; }
        if (row >= 0) write8(y + row * ldy + c * 8, v, cols - c * 8);
    }
}

}  // namespace rgnn
