// typed_linear.hip -- the typed linear over ragged segments whose offsets lie on the
// device: Y[scatter[i]] = X[gather[i]] W[t(i)], weights as stored or transposed (the
// input gradient), and its 8-bit forms.
//
// A workgroup takes BM x BN outputs of one type and walks k in steps of 128 bytes of a row
// (32 fp32, 64 16-bit or 128 8-bit values), which makes one kernel of all types: the same
// rows in LDS, the same loads, and 16-byte chunks that feed the matrix cores in an order of
// k that is the same for both operands.  Steps go straight from memory to LDS (16 bytes a
// lane, no registers), the next one while this one is multiplied.
//
//   Rows of k (X, and W where its k lie side by side): LDS rows of 128 bytes; chunk c of
//     row r lies at position c ^ ((r >> 1) & 7), so that the 16 rows that a fragment reads
//     at one chunk lie in 16 different places of the 64 banks.  The loads write LDS in lane
//     order, so it is their source address that is permuted.
//   Rows of n (W as stored): LDS rows of BN values for each k.  16-bit fragments are read
//     with the transposing LDS read: lane 4 r + c of 16 brings row k = r, columns 4 c, and
//     lane n gets the four k of its column.  Units of 32 bytes are permuted by k so that the
//     eight rows of half a wave lie in different banks.
//
// The product is formed as D[n][m], so that a lane holds four outputs side by side of one
// row; 16-bit rows are turned in LDS and written in pieces as wide as a wave's columns.
//
// What bounds it, and what it measured (copies reach 5.2 TB/s here, large bf16 products 1.1 PFLOP/s):
//   few rows: the weights' bytes, and the latency of the steps (16 rows of 2048 -> 1536, 13 of 32 types'
//     weights read: 19 us, 4.3 TB/s; in 8 bits 10 us, 4.0 TB/s; as integers, 10 of 32 types, 9 us);
//   many rows of narrow weights: memory (300 007 rows 64 -> 64, fp16: 16 us, 5.0 TB/s; 1 000 003
//     gathered and scattered rows 64 -> 128, bf16: 95 us, 4.1 TB/s of rows at random, each counted as often as it is read; rows of
//     8-bit integers in order, codes of 128 bytes, 85 us, 4.6 TB/s);
//   many rows of wide weights: the matrix cores, at the rate of the whole tiles that the types' sizes
//     leave (16 384 rows of 32 types, 2048 -> 4096, bf16: 322 us, 0.85 PFLOP/s; one type 242 us, 1.14; 8
//     bits, 8192 rows 4096 -> 4096: 156 us, 1.76 PFLOP/s; as integers 151 us, 139 in a graph, 1.8 to 2.0 POP/s);
//   thousands of types: the search for a tile, which every workgroup makes from the first offset on (bf16, 65 535
//     rows, 64 -> 64: 1024 types 10 us, 4096 42, 16 384 380, 65 535 5.1 ms).
#include <algorithm>
#include <cmath>

#include "wide_tile.h"

namespace rgnn {

namespace {

struct TileArgs {
    const char *X;
    int64_t x_rows, ldx;         // bytes of a row
    const int32_t *gather;
    const int64_t *ptr;
    int T;
    int64_t M;
    const char *W;
    int64_t w_type, w_row;       // bytes of one type's weights, of one row of them
    int K, N;
    char *Y;
    int64_t y_rows, ldy;         // ldy in elements
    const int32_t *scatter;
    int y_f32, y_f16;            // fp32 outputs; of 8-bit products fp16 ones
    const char *x_end, *w_end;   // behind the last element
    int window;                  // workgroups dealt to the XCDs at a time, over 8
    const uint8_t *xs, *ws;      // fp8: scale bytes
    int ks, nb;                  // bytes of a row's scales; 128-blocks of n
    const float *xf, *wf;        // int8: scales of rows and of outputs
};

struct F8 { typedef uint8_t elem; };

// Each thread of the first BM looks up one row of a tile: which row of X it reads (-1: none of
// them, zeros) and where it goes (-1: nowhere; below -1: zeros go to row -2 - to).  A row outside X
// counts as zeros whatever the weights hold.
__device__ __forceinline__ void tile_row(const TileArgs &a, int64_t i, int64_t end, int &from, int &to)
{
    const int64_t at = min(i, end - 1);             // rows behind the type's: not written
    const int64_t row = a.gather ? (int64_t)a.gather[at] : at, out = a.scatter ? (int64_t)a.scatter[at] : at;
    const bool in = row >= 0 && row < a.x_rows;
    from = in ? (int)row : -1;
    to = i < end && out >= 0 && out < a.y_rows ? (int)out : -1;
    if (!in && to >= 0) to = -2 - to;
}

// int8: the scales of four outputs side by side, of those that the weight has.
__device__ __forceinline__ void output_scales(const TileArgs &a, int type, int j, float (&out)[4])
{
    const float *wf = a.wf + (int64_t)type * a.N;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = wf[min(j + i, a.N - 1)];
}

// ANY: rows on any address.  Loads go through registers (16 bytes from any address; at the end of
// k and of the matrix by elements) and are written to LDS a step later.  STAGES: 1 where all of k is
// one step, which leaves LDS and registers for more workgroups on a CU; 4 where a CU has few of them and
// memory's latency is theirs to bear.  The bounds on registers keep the sums where the products take them, without
// copies, and with one step four workgroups on a CU (1 000 003 gathered rows 64 -> 128: 107 us with three, 98).
template <class T, int BM, int BN, int WM, int WN, bool TRANS, bool ANY, int STAGES>
__global__ __launch_bounds__(WM *WN * 64, STAGES == 1 ? 4 : 2) void typed_linear_kernel(TileArgs a)
{
    typedef typename T::elem E;
    constexpr bool FP8 = std::is_same<T, F8>::value, INT8 = std::is_same<T, I8>::value;
    constexpr int NW = WM * WN, KE = 128 / sizeof(E);
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;     // fragments of a wave
    constexpr int NA = BM / 8 / NW, NB = BN / 8 / NW;       // KB that a wave loads each step
    static_assert(NA * 8 * NW == BM && NB * 8 * NW == BN && NW % 2 == 0 && BM <= NW * 64, "whole loads");
    __shared__ __attribute__((aligned(1024))) char s0[(BM + BN) * 128], s1[STAGES > 1 ? (BM + BN) * 128 : 16];
    __shared__ __attribute__((aligned(1024))) char s2[STAGES > 2 ? (BM + BN) * 128 : 16], s3[STAGES > 2 ? (BM + BN) * 128 : 16];
    __shared__ int from[BM], to[BM];
    char *sa0 = s0, *sb0 = s0 + BM * 128, *sa1 = s1, *sb1 = s1 + (STAGES > 1 ? BM * 128 : 0);
    char *sa2 = s2, *sb2 = s2 + (STAGES > 2 ? BM * 128 : 0), *sa3 = s3, *sb3 = s3 + (STAGES > 2 ? BM * 128 : 0);

    const int nt = (a.N + BN - 1) / BN;
    Piece p;
    if (!find_piece(a.ptr, a.T, a.M, xcd_tile(a.window), [=](int64_t c) { return (c + BM - 1) / BM * nt; }, NoWeight(), p))
        return;
    int mi, ni;
    tile_place(p.index, (int)((p.end - p.begin + BM - 1) / BM), nt, mi, ni);
    const int64_t i0 = p.begin + (int64_t)mi * BM;
    const int j0 = ni * BN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, g = lane >> 4;
    if (threadIdx.x < BM) tile_row(a, i0 + threadIdx.x, p.end, from[threadIdx.x], to[threadIdx.x]);
    __syncthreads();

    // ---- where this lane's loads come from
    const char *zeros = (const char *)&kZeros;
    const char *ap[NA], *bp[NB];
    uint32_t aok = 0;                               // bit x: row x is one of X
    const int chunk = (lane & 7) ^ ((wave & 1) << 2 | lane >> 4);   // of rows of k
#pragma unroll
    for (int x = 0; x < NA; ++x) {
        const int row = from[(x * NW + wave) * 8 + (lane >> 3)];
        ap[x] = row >= 0 ? a.X + row * a.ldx + chunk * 16 : zeros;
        aok |= (row >= 0 ? 1u : 0u) << x;
    }
    const char *W = a.W + (int64_t)p.type * a.w_type;
    int bk[NB];                                     // rows of n: the k of the load
    const int64_t binc = TRANS ? 128 : KE * a.w_row;
#pragma unroll
    for (int x = 0; x < NB; ++x) {
        if (TRANS) {
            const int j = min(j0 + (x * NW + wave) * 8 + (lane >> 3), a.N - 1);
            bp[x] = W + j * a.w_row + chunk * 16;
            bk[x] = 0;
        } else {
            constexpr int CH = BN * sizeof(E) / 16, UC = sizeof(E) == 4 ? 4 : 2;   // chunks of a row, of a unit
            const int at = (x * NW + wave) * 64 + lane, k = at / CH, pos = at % CH;
            const int c = (pos / UC ^ unit_turn<T, BN>(k)) * UC + pos % UC;
            const int j = j0 + c * (16 / (int)sizeof(E));
            bk[x] = k;
            bp[x] = W + k * a.w_row + (j < a.N ? j : 0) * (int64_t)sizeof(E);
        }
    }
    const int kbytes = a.K * (int)sizeof(E);
    const int steps = (kbytes + 127) / 128;
    auto load = [&](char *sa, char *sb, int step) {
        const bool tail = (step + 1) * 128 > kbytes;
#pragma unroll
        for (int x = 0; x < NA; ++x) {
            const char *src = tail && step * 128 + chunk * 16 >= kbytes ? zeros : ap[x];
            load_lds(src, sa + (x * NW + wave) * 1024);
            ap[x] += (aok >> x & 1) << 7;
        }
#pragma unroll
        for (int x = 0; x < NB; ++x) {
            const bool out = TRANS ? step * 128 + chunk * 16 >= kbytes : step * KE + bk[x] >= a.K;
            load_lds(tail && out ? zeros : bp[x], sb + (x * NW + wave) * 1024);
            bp[x] += binc;
        }
    };
    // ANY: a step's loads into registers, and from there to LDS.  Several steps are under way (SETS).
    constexpr int SETS = !ANY || STAGES == 1 ? 1 : NA + NB <= 6 ? 4 : 2;
    struct Set { i32x4 a[ANY ? NA : 1], b[ANY ? NB : 1]; } set[SETS];
    auto fetch = [&](Set &r, int step) {
        if constexpr (ANY) {
            const int left = kbytes - step * 128 - chunk * 16;   // bytes of k from this chunk on
#pragma unroll
            for (int x = 0; x < NA; ++x) {
                r.a[x] = left > 0 && (aok >> x & 1) ? load_any<E>(ap[x], a.x_end) : i32x4{0, 0, 0, 0};
                ap[x] += (aok >> x & 1) << 7;
            }
#pragma unroll
            for (int x = 0; x < NB; ++x) {
                const bool in = TRANS ? left > 0 : step * KE + bk[x] < a.K;
                r.b[x] = in ? load_any<E>(bp[x], a.w_end) : i32x4{0, 0, 0, 0};
                bp[x] += binc;
            }
        }
    };
    auto put = [&](Set &r, char *sa, char *sb, int step) {
        if constexpr (ANY) {
            if ((step + 1) * 128 > kbytes) {        // here, not at the load: nothing is to wait for it before
                const int left = kbytes - step * 128 - chunk * 16;
#pragma unroll
                for (int x = 0; x < NA; ++x) r.a[x] = first_bytes(r.a[x], left);
                if (TRANS)
#pragma unroll
                    for (int x = 0; x < NB; ++x) r.b[x] = first_bytes(r.b[x], left);
            }
#pragma unroll
            for (int x = 0; x < NA; ++x) *(i32x4 *)(sa + (x * NW + wave) * 1024 + lane * 16) = r.a[x];
#pragma unroll
            for (int x = 0; x < NB; ++x) *(i32x4 *)(sb + (x * NW + wave) * 1024 + lane * 16) = r.b[x];
        }
    };

    // ---- where its fragments lie
    const int wm = wave / WN, wn = wave % WN;
    const int turn = (r16 >> 1) & 7;
    int aoff[2], boff[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) aoff[q] = (wm * FM * 16 + r16) * 128 + (((g + 4 * q) ^ turn) * 16);
#pragma unroll
    for (int q = 0; q < 2; ++q) boff[q] = (wn * FN * 16 + r16) * 128 + (((g + 4 * q) ^ turn) * 16);
    int uoff[FN];                                   // rows of n
    if (!TRANS) {
        if (sizeof(E) == 2) {
            const int r = (lane & 15) >> 2, c = lane & 3, k = g * 8 + r;
#pragma unroll
            for (int f = 0; f < FN; ++f) uoff[f] = k * BN * 2 + ((wn * FN + f) ^ unit_turn<T, BN>(k)) * 32 + c * 8;
        } else {
#pragma unroll
            for (int f = 0; f < FN; ++f) uoff[f] = g * 4 * BN * 4 + ((wn * FN + f) ^ g) * 64 + r16 * 4;
        }
    }
    f32x4 acc[FM][FN] = {};

    // int8: the scales of this lane's rows and outputs, on their way before the steps.  The one-step 128 x 128 tile, whose
    // bound on registers leaves no room for them beside its sums, reads them afterwards (before, 20 registers spilled: 1 000 003 rows
    // 64 -> 128 113 us, 85 now; 300 007 rows of 96 types 128 -> 128 35 and 26; but 64 -> 64, 128 x 64 tiles, 16.8 before, 18.2 after).
    constexpr bool BEFORE = STAGES > 1 || FM * FN < 16;
    float xf[INT8 ? FM : 1], wf[INT8 ? FN : 1][4];
    auto factors = [&] {
        if constexpr (INT8) {
#pragma unroll
            for (int m = 0; m < FM; ++m) {
                const int row = from[(wm * FM + m) * 16 + r16];
                xf[m] = *(const float *)(row >= 0 ? (const char *)(a.xf + row) : zeros);
            }
#pragma unroll
            for (int f = 0; f < FN; ++f) output_scales(a, p.type, j0 + (wn * FN + f) * 16 + g * 4, wf[f]);
        }
    };
    if (BEFORE) factors();

    // fp8: the scale bytes of this lane's rows and of the weights, whose columns of a wave lie in one
    // block of 128.  A word is four steps; the next one is read a word ahead.
    const char *xs[FP8 ? FM : 1];
    const uint8_t *wp = nullptr;
    int sx[FP8 ? FM : 1], nx[FP8 ? FM : 1], sw = 0, nw = 0;
    uint32_t xin = 0;
    if constexpr (FP8) {
        static_assert(FN * 16 <= 128 && 128 % (FN * 16) == 0, "scales");
#pragma unroll
        for (int m = 0; m < FM; ++m) {
            const int row = from[(wm * FM + m) * 16 + r16];
            xs[m] = row >= 0 ? (const char *)a.xs + (int64_t)row * a.ks : zeros;
            xin |= (row >= 0 ? 4u : 0u) << m * 3;
            nx[m] = *(const __attribute__((address_space(1))) int *)xs[m];
        }
        wp = a.ws + ((int64_t)p.type * a.nb + min(j0 + wn * FN * 16, a.N - 1) / 128) * a.ks;
        nw = *(const int *)wp;
    }
    auto scales = [&](int step) {
        if constexpr (FP8) {
            if ((step & 3) == 0) {
                sw = nw;
#pragma unroll
                for (int m = 0; m < FM; ++m) sx[m] = nx[m];
                if (step + 4 < a.ks) {
                    nw = *(const int *)(wp + step + 4);
#pragma unroll
                    for (int m = 0; m < FM; ++m) {
                        xs[m] += xin >> m * 3 & 4;
                        nx[m] = *(const __attribute__((address_space(1))) int *)xs[m];
                    }
                }
            }
        }
    };
    auto multiply = [&](const char *sa, const char *sb) {
        if constexpr (FP8) {
            i32x8 fb[FN];
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                const i32x4 x = *(const i32x4 *)(sb + boff[0] + f * 2048), y = *(const i32x4 *)(sb + boff[1] + f * 2048);
                fb[f] = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
            }
#pragma unroll
            for (int m = 0; m < FM; ++m) {
                const i32x4 x = *(const i32x4 *)(sa + aoff[0] + m * 2048), y = *(const i32x4 *)(sa + aoff[1] + m * 2048);
                const i32x8 fa = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int f = 0; f < FN; ++f)
                    acc[m][f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[f], fa, acc[m][f], 0, 0, 0, sw, 0, sx[m]);
            }
#pragma unroll
            for (int f = 0; f < FM; ++f) sx[f] = (int)((uint32_t)sx[f] >> 8);
            sw = (int)((uint32_t)sw >> 8);
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                __builtin_amdgcn_sched_barrier(0);
                i32x4 fb[FN], fa[FM];
#pragma unroll
                for (int f = 0; f < FN; ++f) {
                    if constexpr (TRANS) fb[f] = *(const i32x4 *)(sb + boff[q] + f * 2048);
                    else if constexpr (sizeof(E) == 2) {
                        const uint64_t x = read_turned(sb + uoff[f] + q * 32 * BN * 2);
                        const uint64_t y = read_turned(sb + uoff[f] + (q * 32 + 4) * BN * 2);
                        fb[f] = i32x4{(int)x, (int)(x >> 32), (int)y, (int)(y >> 32)};
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) fb[f][i] = *(const int *)(sb + uoff[f] + (q * 16 + i) * BN * 4);
                    }
                }
#pragma unroll
                for (int m = 0; m < FM; ++m) fa[m] = *(const i32x4 *)(sa + aoff[q] + m * 2048);
#pragma unroll
                for (int m = 0; m < FM; ++m)
#pragma unroll
                    for (int f = 0; f < FN; ++f) acc[m][f] = mma16<T>(fb[f], fa[m], acc[m][f]);
            }
        }
    };

    int step = 0;
    if constexpr (STAGES == 1) {
        if constexpr (ANY) {
            fetch(set[0], 0);
            put(set[0], sa0, sb0, 0);
        } else {
            load(sa0, sb0, 0);
        }
        step_barrier<0>();
        scales(0);
        multiply(sa0, sb0);
    } else if constexpr (STAGES == 4) {
        // three steps under way, in whole rounds of four: what lies behind K is zeros
        constexpr int ONE = NA + NB;
        load(sa0, sb0, 0);
        load(sa1, sb1, 1);
        load(sa2, sb2, 2);
        for (; step + 4 < steps; step += 4) {
            step_barrier<2 * ONE>();
            load(sa3, sb3, step + 3);
            scales(step);
            multiply(sa0, sb0);
            step_barrier<2 * ONE>();
            load(sa0, sb0, step + 4);
            multiply(sa1, sb1);
            step_barrier<2 * ONE>();
            load(sa1, sb1, step + 5);
            multiply(sa2, sb2);
            step_barrier<2 * ONE>();
            load(sa2, sb2, step + 6);
            multiply(sa3, sb3);
        }
        step_barrier<2 * ONE>();
        load(sa3, sb3, step + 3);
        scales(step);
        multiply(sa0, sb0);
        step_barrier<2 * ONE>();
        multiply(sa1, sb1);
        step_barrier<ONE>();
        multiply(sa2, sb2);
        step_barrier<0>();
        multiply(sa3, sb3);
    } else if constexpr (ANY) {
        // whole rounds of SETS steps; those behind K are zeros
#pragma unroll
        for (int u = 0; u < SETS; ++u) fetch(set[u], u);
        put(set[0], sa0, sb0, 0);
        fetch(set[0], SETS);
        for (; step < steps; step += SETS) {
#pragma unroll
            for (int u = 0; u < SETS; ++u) {
                __syncthreads();
                multiply(u & 1 ? sa1 : sa0, u & 1 ? sb1 : sb0);
                Set &next = set[(u + 1) % SETS];
                put(next, u & 1 ? sa0 : sa1, u & 1 ? sb0 : sb1, step + u + 1);
                fetch(next, step + u + 1 + SETS);
            }
        }
    } else {
        load(sa0, sb0, 0);
        for (; step + 2 <= steps; step += 2) {
            step_barrier<0>();
            scales(step);
            load(sa1, sb1, step + 1);
            multiply(sa0, sb0);
            step_barrier<0>();
            if (step + 2 < steps) load(sa0, sb0, step + 2);
            multiply(sa1, sb1);
        }
        if (step < steps) {
            step_barrier<0>();
            scales(step);
            multiply(sa0, sb0);
        }
    }

    // ---- write
    const int *out = to + wm * FM * 16;
    const int j1 = j0 + wn * FN * 16;               // this wave's first column
    if constexpr (INT8) {                           // whole numbers to fp32, times the scales
        if (!BEFORE) factors();
#pragma unroll
        for (int m = 0; m < FM; ++m)
#pragma unroll
            for (int f = 0; f < FN; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][f][i] = (float)__float_as_int(acc[m][f][i]) * xf[m] * wf[f][i];
    }
    if (sizeof(E) == 4 || a.y_f32) {
#pragma unroll
        for (int m = 0; m < FM; ++m) {
            int row = out[m * 16 + r16];
            const bool zero = row < -1;
            if (zero) row = -2 - row;
            if (row < 0) continue;
#pragma unroll
            for (int f = 0; f < FN; ++f) {
                const int j = j1 + f * 16 + g * 4;
                write4((float *)a.Y + row * a.ldy + j, zero ? f32x4{0, 0, 0, 0} : acc[m][f], a.N - j);
            }
        }
        return;
    }
    step_barrier<0>();                              // the stages may be used again
    char *mine = s0 + wave * (FM * FN * 512);
    if (sizeof(E) == 1 && a.y_f16) write_rows<_Float16, FM, FN>(mine, acc, (_Float16 *)a.Y + j1, a.ldy, a.N - j1, lane, out);
    else write_rows<typename std::conditional<sizeof(E) != 2, __bf16, E>::type, FM, FN>(
        mine, acc, (typename std::conditional<sizeof(E) != 2, __bf16, E>::type *)a.Y + j1, a.ldy, a.N - j1, lane, out);
}

// The wide tile (wide_tile.h).  A tile with at most half of its rows does half the work.
template <class T, bool TRANS>
__global__ __launch_bounds__(256, 1) void typed_linear_wide_kernel(TileArgs a)
{
    typedef typename T::elem E;
    constexpr bool FP8 = std::is_same<T, F8>::value, INT8 = std::is_same<T, I8>::value;
    constexpr int KE = kWideKB / sizeof(E);
    __shared__ __attribute__((aligned(1024))) char s0[2 * kWideStage], s1[2 * kWideStage], s2[2 * kWideStage], s3[2 * kWideStage];
    char *a0 = s0, *b0 = s0 + kWideStage, *a1 = s1, *b1 = s1 + kWideStage;
    char *a2 = s2, *b2 = s2 + kWideStage, *a3 = s3, *b3 = s3 + kWideStage;

    const int nt = (a.N + kWide - 1) / kWide;
    Piece p;
    if (!find_piece(a.ptr, a.T, a.M, xcd_tile(a.window), [=](int64_t c) { return (c + kWide - 1) / kWide * nt; },
                    NoWeight(), p))
        return;
    int mi, ni;
    tile_place((int)p.index, (int)((p.end - p.begin + kWide - 1) / kWide), nt, mi, ni);
    const int64_t i0 = p.begin + (int64_t)mi * kWide;
    const int j0 = ni * kWide;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;

    // the rows' places in 32 bits of bytes from `X` on
    __shared__ int from[kWide], to[kWide];
    const char *X = a.gather ? a.X : a.X + i0 * a.ldx;
    {
        int row;
        tile_row(a, i0 + threadIdx.x, p.end, row, to[threadIdx.x]);
        from[threadIdx.x] = max(0, a.gather ? row : row - (int)i0);   // of zeros: any row
    }
    __syncthreads();
    WideSide sa, sb;
    const int chunk = (lane & 3) ^ wide_turn_k(wave * 16 + (lane >> 2));   // of rows of k
    sa.base = X;
    sa.step = kWideKB;
#pragma unroll
    for (int x = 0; x < kWideLoads; ++x)
        sa.off[x] = (uint32_t)(from[x * 64 + wave * 16 + (lane >> 2)] * a.ldx) + chunk * 16;
    sb.base = a.W + (int64_t)p.type * a.w_type + (TRANS ? j0 * a.w_row : j0 * (int64_t)sizeof(E));
    sb.step = TRANS ? kWideKB : KE * a.w_row;
#pragma unroll
    for (int x = 0; x < kWideLoads; ++x) {
        if (TRANS) {
            const int j = min(x * 64 + wave * 16 + (lane >> 2), a.N - 1 - j0);
            sb.off[x] = (uint32_t)(j * a.w_row) + chunk * 16;
        } else {
            const int k = x * 8 + wave * 2 + (lane >> 5), pos = lane & 31;
            const int j = ((pos >> 1 ^ wide_turn_n(k)) * 2 + (pos & 1)) * 8;
            sb.off[x] = (uint32_t)(k * a.w_row) + (j0 + j < a.N ? j : 0) * (uint32_t)sizeof(E);
        }
    }
    const int kbytes = a.K * (int)sizeof(E);
    const int whole = kbytes / kWideKB, steps = (kbytes + kWideKB - 1) / kWideKB;

    WideFragments<false> fa;
    WideFragments<!TRANS> fb;
    fb.init(wn * 128, lane);

    f32x16 acc[4][4] = {};
    auto walk = [&](auto fm) {
        constexpr int FMV = decltype(fm)::value, LA = kWideLoads * FMV / 4;
        fa.init(wm * FMV * 32, lane);
        // fp8: the scale bytes of this lane's rows, a word is eight steps
        uint32_t xoff[FP8 ? FMV : 1], sx[FP8 ? FMV : 1], nx[FP8 ? FMV : 1], sw = 0, nw = 0;
        const uint8_t *xs = nullptr, *wp = nullptr;
        if constexpr (FP8) {
            xs = a.gather ? a.xs : a.xs + i0 * a.ks;
#pragma unroll
            for (int m = 0; m < FMV; ++m) {
                xoff[m] = (uint32_t)(from[(wm * FMV + m) * 32 + (lane & 31)] * (int64_t)a.ks);
                nx[m] = *(const uint32_t *)(xs + xoff[m]);
            }
            wp = a.ws + ((int64_t)p.type * a.nb + min(j0 + wn * 128, a.N - 1) / 128) * a.ks;
            nw = *(const uint32_t *)wp;
        }
        auto load = [&](char *ta, char *tb) {
            sa.load<LA>(ta, wave);
            sb.load<kWideLoads>(tb, wave);
            sa.base += sa.step;
            sb.base += sb.step;
        };
        auto edge = [&](char *ta, char *tb, int step) {
            if (step < whole) return load(ta, tb);
            const bool in = step * kWideKB + chunk * 16 < kbytes;
            sa.load_edge<LA>(ta, wave, [&](int) { return in; });
            sb.load_edge<kWideLoads>(tb, wave, [&](int x) {
                return TRANS ? in : step * KE + x * 8 + wave * 2 + (lane >> 5) < a.K;
            });
        };
        auto shift = [&](int step) {
            if constexpr (FP8) {
                if ((step & 7) == 0) {              // the next word is read eight steps ahead
#pragma unroll
                    for (int m = 0; m < FMV; ++m) sx[m] = nx[m];
                    sw = nw;
                    const int next = step / 2 + 4;
                    if (next < a.ks) {
#pragma unroll
                        for (int m = 0; m < FMV; ++m) nx[m] = *(const uint32_t *)(xs + next + xoff[m]);
                        nw = *(const uint32_t *)(wp + next);
                    }
                } else if ((step & 1) == 0) {
#pragma unroll
                    for (int m = 0; m < FMV; ++m) sx[m] >>= 8;
                    sw >>= 8;
                }
            }
        };
        auto multiply = [&](const i32x8 (&x)[FMV], const i32x8 (&w)[4], f32x16 (&c)[4][4]) {
            if constexpr (FP8) {
#pragma unroll
                for (int m = 0; m < FMV; ++m)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        c[m][n] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[n], x[m], c[m][n], 0, 0, 0, (int)sw, 0, (int)sx[m]);
                    }
            } else {
#pragma unroll
                for (int q = 0; q < 2; ++q)
#pragma unroll
                    for (int m = 0; m < FMV; ++m)
#pragma unroll
                        for (int n = 0; n < 4; ++n) c[m][n] = mma32<T>(chunk_of(w[n], q), chunk_of(x[m], q), c[m][n]);
            }
        };
        wide_walk<FMV, false, !TRANS, LA + kWideLoads>(a0, b0, a1, b1, a2, b2, a3, b3, fa, fb, steps, whole, load, edge, multiply,
                                                       shift, acc);
        if constexpr (INT8) {
            const float *xf = a.gather ? a.xf : a.xf + i0;
            float x[FMV];
#pragma unroll
            for (int m = 0; m < FMV; ++m) x[m] = xf[from[(wm * FMV + m) * 32 + (lane & 31)]];
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float wf[4];
                    output_scales(a, p.type, j0 + wn * 128 + n * 32 + q * 8 + (lane >> 5) * 4, wf);
#pragma unroll
                    for (int m = 0; m < FMV; ++m)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            acc[m][n][q * 4 + i] = (float)__float_as_int(acc[m][n][q * 4 + i]) * x[m] * wf[i];
                }
        }
        typedef typename std::conditional<sizeof(E) == 1, __bf16, E>::type O;
        const int *out = to + wm * FMV * 32;
        char *mine = wave == 0 ? s0 : wave == 1 ? s1 : wave == 2 ? s2 : s3;
        const int cols = a.N - j0 - wn * 128;
        if (sizeof(E) == 1 && a.y_f16) return wide_write<_Float16, FMV>(mine, acc, (_Float16 *)a.Y + j0 + wn * 128, a.ldy, cols, lane, out);
        if (!a.y_f32) return wide_write<O, FMV>(mine, acc, (O *)a.Y + j0 + wn * 128, a.ldy, cols, lane, out);
#pragma unroll
        for (int m = 0; m < FMV; ++m) {
            int row = out[m * 32 + (lane & 31)];
            const bool zero = row < -1;
            if (zero) row = -2 - row;
            if (row < 0) continue;
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int j = j0 + wn * 128 + n * 32 + q * 8 + (lane >> 5) * 4;
                    f32x4 v = {acc[m][n][q * 4], acc[m][n][q * 4 + 1], acc[m][n][q * 4 + 2], acc[m][n][q * 4 + 3]};
                    if (zero) v = f32x4{0, 0, 0, 0};
                    write4((float *)a.Y + row * a.ldy + j, v, a.N - j);
                }
        }
    };
    if (p.end - i0 <= kWide / 2) walk(std::integral_constant<int, 2>());
    else walk(std::integral_constant<int, 4>());
}

template <class T, bool TRANS>
rgnn_status launch_wide(TileArgs k, hipStream_t s)
{
    const int64_t tiles = row_tiles_bound(k.M, k.T, kWide) * ((k.N + kWide - 1) / kWide);
    k.window = xcd_window(tiles);
    const int64_t grid = xcd_grid(tiles, k.window);
    if (grid >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many tiles");
    hipLaunchKernelGGL((typed_linear_wide_kernel<T, TRANS>), flat_grid(grid), dim3(256), 0, s, k);
    return RGNN_OK;
}

template <class T, int BM, int BN, int WM, int WN, bool TRANS, bool ANY, bool DEEP = false>
rgnn_status launch_tile(TileArgs k, hipStream_t s)
{
    const int64_t tiles = row_tiles_bound(k.M, k.T, BM) * ((k.N + BN - 1) / BN);
    k.window = xcd_window(tiles);
    const int64_t grid = xcd_grid(tiles, k.window);
    if (grid >= (int64_t(1) << 31)) return fail(RGNN_ERANGE, "too many tiles");
    const dim3 g = flat_grid(grid), b(WM * WN * 64);
    if constexpr (DEEP)              // of many steps
        hipLaunchKernelGGL((typed_linear_kernel<T, BM, BN, WM, WN, TRANS, ANY, 4>), g, b, 0, s, k);
    else if (k.K * (int)sizeof(typename T::elem) <= 128)
        hipLaunchKernelGGL((typed_linear_kernel<T, BM, BN, WM, WN, TRANS, ANY, 1>), g, b, 0, s, k);
    else
        hipLaunchKernelGGL((typed_linear_kernel<T, BM, BN, WM, WN, TRANS, ANY, 2>), g, b, 0, s, k);
    return RGNN_OK;
}

// Which tile of 16 and 8 bits: each is priced and the cheapest is taken.  The prices were fitted to times in us (1 to
// 16384 rows, k of 512 to 4096, one to 32 types, mostly 16 bits) and tell which tile is faster, not how long
// it takes: kernels take 1.05 to 1.6 times theirs (16 rows of 32 types, 2048 -> 1536: priced 11.8, takes 18.8; in 8 bits 6.9
// and 10.2; 8192 rows, 4096 -> 4096, 8 bits: 120 and 156).  `slots` workgroups fit the chip; a round of them
// costs `each` and, for each KB of k of a row, `full`, down to `light` where few of the slots are taken.  Where
// a CU has several slots, rounds run into each other: a last one in part costs half as if it were apart and
// half its share (8192 rows of 16 types, 1536 -> 2048, bf16: 128 x 128, 2.25 rounds, 68 us; 128 x 64, 3, 75; 256 x 256,
// 1.25, 81).
// The deep ones, with four stages, are for few tiles (64 rows, 4096 x 4096, bf16: 32 x 64 17 us, 64 x 64
// 20, 128 x 64 with two stages 36; 1024 rows 76, 58 and 47).  Rows on any address wait for registers at
// each step: theirs are priced apart (bf16; 292 rows, 1561 -> 333: 32 x 64 17 us, 128 x 64 30, 128 x 128 37; 8192
// rows, 2047 -> 1535: 209, 119 and 93; 300 007 rows of 96 types, 61 -> 61: 27, 22 and 24).
struct TileCost {
    int bm, bn, slots;
    double each, light, full;
};
constexpr TileCost kCostWide = {256, 256, 256, 9.0, 7.0, 12.8};
constexpr TileCost kCost128 = {128, 128, 512, 3.0, 6.0, 8.5};
constexpr TileCost kCostNarrow = {128, 64, 768, 2.5, 3.7, 7.5};
constexpr TileCost kCostDeep = {64, 64, 512, 2.0, 1.9, 3.3};
constexpr TileCost kCostDeepSmall = {32, 64, 768, 2.0, 1.6, 3.3};
constexpr TileCost kAnyCost128 = {128, 128, 512, 4.0, 9.0, 14.0};
constexpr TileCost kAnyCostNarrow = {128, 64, 768, 3.5, 8.5, 13.5};
constexpr TileCost kAnyCostSmall = {32, 64, 768, 2.5, 4.6, 7.0};

// Tiles that the rows make: every type that has some leaves half a tile, and has one at least.
double tiles_of(const TileArgs &k, int bm, int bn)
{
    const double types = (double)std::min<int64_t>(k.M, k.T);
    const double rows = types == 1 ? std::ceil((double)k.M / bm) : std::max((double)k.M / bm + types / 2, types);
    return rows * ((k.N + bn - 1) / bn);
}

double tile_cost(const TileArgs &k, const TileCost &c, int el)
{
    const double tiles = tiles_of(k, c.bm, c.bn), kb = (double)k.K * el / 1024;
    const double rounds = std::floor(tiles / c.slots), rest = tiles / c.slots - rounds;
    const double round = c.each + c.full * kb, last = rest > 0 ? c.each + (c.light + (c.full - c.light) * rest) * kb : 0;
    return rounds * round + (rounds > 0 && c.slots > 256 ? (last + rest * round) / 2 : last);
}

// The tile of a call; el: bytes of an element, any: rows on any address.
enum class Shape { k32x64, k32x64Deep, k64x64, k64x64Deep, k128x64, k128x128, kWide };

// fp32 is bound by its matrix cores, which take as long for a tile of few rows as for a full one: 64 x 64
// where those give every CU two, 32 x 64 below (33 rows of 7 types, 2624 -> 128: 38 us, 64 x 64 59,
// 128 x 128 182; 600 000 rows 128 -> 128: 294, 253).  Four stages from 16 steps of k on (1816 -> 1192:
// 26-29 us, with two 30; 5 steps 13, with two 11).
Shape choose_tile(const TileArgs &k, int el, bool any)
{
    if (el == 4) {
        if (tiles_of(k, 64, 64) >= 512) return Shape::k64x64;
        return !any && k.K >= 512 ? Shape::k32x64Deep : Shape::k32x64;
    }
    if (any) {
        const double small = tile_cost(k, kAnyCostSmall, el), narrow = tile_cost(k, kAnyCostNarrow, el), c128 = tile_cost(k, kAnyCost128, el);
        if (small < std::min(narrow, c128)) return Shape::k32x64;
        return narrow <= c128 ? Shape::k128x64 : Shape::k128x128;
    }
    const double narrow = tile_cost(k, kCostNarrow, el), c128 = tile_cost(k, kCost128, el), wide = tile_cost(k, kCostWide, el);
    const double best = std::min(narrow, c128);
    // the wide tile's offsets have 32 bits
    const bool near = k.x_rows > 0 && (k.gather ? k.x_rows : (int64_t)kWide) * k.ldx < (int64_t(1) << 32) &&
                      kWide * k.w_row < (int64_t(1) << 32);
    if (k.K * el > 128) {      // more than one step
        const double deep = tile_cost(k, kCostDeep, el), small = tile_cost(k, kCostDeepSmall, el);
        if (small < std::min(deep, best)) return Shape::k32x64Deep;
        if (deep < best && !(near && wide < deep)) return Shape::k64x64Deep;
    }
    if (near && wide < best) return Shape::kWide;
    return narrow <= c128 ? Shape::k128x64 : Shape::k128x128;
}

template <class T, bool TRANS, bool ANY>
rgnn_status launch_shape(const TileArgs &k, hipStream_t s)
{
    constexpr int el = sizeof(typename T::elem);
    const Shape tile = choose_tile(k, el, ANY);
    if constexpr (el == 4) {
        if (tile == Shape::k64x64) return launch_tile<F32, 64, 64, 2, 2, TRANS, ANY>(k, s);
        if constexpr (!ANY)
            if (tile == Shape::k32x64Deep) return launch_tile<F32, 32, 64, 2, 2, TRANS, false, true>(k, s);
        return launch_tile<F32, 32, 64, 2, 2, TRANS, ANY>(k, s);
    } else {
        if constexpr (ANY) {
            if (tile == Shape::k32x64) return launch_tile<T, 32, 64, 2, 2, TRANS, true>(k, s);
        } else {
            if (tile == Shape::k32x64Deep) return launch_tile<T, 32, 64, 2, 2, TRANS, false, true>(k, s);
            if (tile == Shape::k64x64Deep) return launch_tile<T, 64, 64, 2, 2, TRANS, false, true>(k, s);
            if (tile == Shape::kWide) return launch_wide<T, TRANS>(k, s);
        }
        if (tile == Shape::k128x64) return launch_tile<T, 128, 64, 4, 1, TRANS, ANY>(k, s);
        return launch_tile<T, 128, 128, 2, 2, TRANS, ANY>(k, s);
    }
}

TileArgs tile_args(const LinearArgs &a)
{
    const int el = dtype_bytes(a.dtype);
    TileArgs k{};
    k.X = (const char *)a.X; k.x_rows = a.x_rows; k.ldx = a.ldx * el; k.gather = a.gather;
    k.ptr = a.type_ptr; k.T = a.T; k.M = a.M;
    k.W = (const char *)a.W; k.K = a.K; k.N = a.N;
    k.w_row = (int64_t)(a.trans_w ? a.K : a.N) * el;
    k.w_type = (int64_t)a.K * a.N * el;
    k.Y = (char *)a.Y; k.y_rows = a.y_rows; k.ldy = a.ldy; k.scatter = a.scatter;
    k.y_f32 = a.y_dtype == RGNN_F32;
    k.x_end = k.X + ((a.x_rows - 1) * a.ldx + a.K) * el;
    k.w_end = k.W + a.T * k.w_type;
    return k;
}

// Whole vectors of 16 bytes in every row go straight to LDS.
bool whole_rows(const LinearArgs &a)
{
    const int el = dtype_bytes(a.dtype);
    return (uintptr_t)a.X % 16 == 0 && (uintptr_t)a.W % 16 == 0 && a.ldx * el % 16 == 0 && (int64_t)a.K * el % 16 == 0 &&
           (int64_t)a.N * el % 16 == 0;
}

TileArgs tile_args_eight(const LinearArgs &a)
{
    TileArgs k = tile_args(a);
    k.K = fp8_width(a.K);
    k.w_row = k.K; k.w_type = (int64_t)k.K * a.N;
    k.xs = a.x_scale; k.ws = a.w_scale; k.ks = fp8_scales(a.K); k.nb = (a.N + 127) / 128;
    k.xf = a.x_factor; k.wf = a.w_factor;
    k.y_f16 = a.y_dtype == RGNN_F16;
    return k;
}

template <class T>
rgnn_status launch_type(const TileArgs &k, int trans, bool whole, hipStream_t s)
{
    if (whole) return trans ? launch_shape<T, true, false>(k, s) : launch_shape<T, false, false>(k, s);
    return trans ? launch_shape<T, true, true>(k, s) : launch_shape<T, false, true>(k, s);
}

}  // namespace

rgnn_tile_t typed_linear_tile(const LinearArgs &a)
{
    const bool eight = dtype_eight(a.dtype), any = !eight && !whole_rows(a);
    const TileArgs k = eight ? tile_args_eight(a) : tile_args(a);
    const int el = dtype_bytes(a.dtype), one = k.K * el <= 128 ? 1 : 0;
    switch (choose_tile(k, el, any)) {
    case Shape::k32x64: return {32, 64, one ? 1 : 2, any};
    case Shape::k32x64Deep: return {32, 64, one ? 1 : 4, any};
    case Shape::k64x64: return {64, 64, one ? 1 : 2, any};
    case Shape::k64x64Deep: return {64, 64, one ? 1 : 4, any};
    case Shape::k128x64: return {128, 64, one ? 1 : 2, any};
    case Shape::k128x128: return {128, 128, one ? 1 : 2, any};
    default: return {kWide, kWide, 4, any};
    }
}

rgnn_status launch_typed_linear(const LinearArgs &a, hipStream_t s)
{
    const bool whole = whole_rows(a);
    const TileArgs k = tile_args(a);
    rgnn_status st;
    {
        LaunchScope ls("typed_linear", s);
        if (a.dtype == RGNN_F32) st = launch_type<F32>(k, a.trans_w, whole, s);
        else if (a.dtype == RGNN_BF16) st = launch_type<BF16>(k, a.trans_w, whole, s);
        else st = launch_type<F16>(k, a.trans_w, whole, s);
    }
    if (st != RGNN_OK) return st;
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "typed_linear launch");
}

rgnn_status launch_typed_fp8(const LinearArgs &a, hipStream_t s)
{
    const TileArgs k = tile_args_eight(a);
    rgnn_status st;
    {
        LaunchScope ls("typed_linear_fp8", s);
        st = launch_shape<F8, true, false>(k, s);
    }
    if (st != RGNN_OK) return st;
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "typed_linear_fp8 launch");
}

rgnn_status launch_typed_int8(const LinearArgs &a, hipStream_t s)
{
    const TileArgs k = tile_args_eight(a);
    rgnn_status st;
    {
        LaunchScope ls("typed_linear_int8", s);
        st = launch_shape<I8, true, false>(k, s);
    }
    if (st != RGNN_OK) return st;
    hipError_t e = hipGetLastError();
    return e == hipSuccess ? RGNN_OK : hip_fail(e, "typed_linear_int8 launch");
}

}  // namespace rgnn
