"""Every tile of the typed linear, its 8-bit form and its weight gradient against 64 bits.

The tile is chosen by a price, so a test of given sizes may come to run another one when prices change:
each case here names the tile that it is for, and asks for it (on the CPU too).

Rows are ragged: types of no row, of one, of up to half a wide tile and of more, positions of no type on both
sides.  K ends inside a step, N inside a tile (or a wave's part of one lies outside).  Tolerances are those of
test_linear_ops.py; they grow with the number of summands, so small integers, whose sums fp32 holds exactly, are
multiplied too and have to come out to the bit: no row or column is left out or taken twice."""
import math

import numpy as np
import pytest

from test_linear_ops import GROUPED, close, fp8_values, linear_ref, types, wgrad_ref, workspace

gpu = pytest.mark.gpu

SIZES = [600, 1, 0, 1256, 300, 127, 215]
BEFORE, BEHIND = 5, 9
M = BEFORE + sum(SIZES) + BEHIND
PTR = [BEFORE] + (BEFORE + np.cumsum(SIZES)).tolist()
T = len(SIZES)

# K, N, the tile: rows, columns, stages, any address
TILES_16 = [
    (40, 1288, (128, 64, 1, False)), (72, 1288, (128, 64, 2, False)), (520, 2056, (128, 64, 2, False)),
    (56, 2200, (128, 128, 1, False)), (72, 2200, (128, 128, 2, False)), (520, 4104, (128, 128, 2, False)),
    (72, 648, (64, 64, 4, False)), (1000, 1000, (64, 64, 4, False)),
    (72, 136, (32, 64, 4, False)), (1096, 136, (32, 64, 4, False)),
    (1000, 4104, (256, 256, 4, False)), (1096, 4240, (256, 256, 4, False)), (1024, 4096, (256, 256, 4, False)),
    (33, 301, (32, 64, 1, True)), (777, 150, (32, 64, 2, True)),
    (33, 777, (128, 64, 1, True)), (303, 1301, (128, 64, 2, True)),
    (33, 2501, (128, 128, 1, True)), (303, 2501, (128, 128, 2, True)), (777, 2501, (128, 128, 2, True)),
]
TILES_32 = [
    (16, 136, (32, 64, 1, False)), (100, 328, (32, 64, 2, False)), (520, 328, (32, 64, 4, False)),
    (28, 1000, (64, 64, 1, False)), (520, 1000, (64, 64, 2, False)),
    (30, 301, (32, 64, 1, True)), (303, 301, (32, 64, 2, True)), (31, 777, (64, 64, 1, True)), (303, 777, (64, 64, 2, True)),
]
TILES_8 = [
    (100, 1288, (128, 64, 1, False)), (700, 1288, (128, 64, 2, False)),
    (100, 2200, (128, 128, 1, False)), (200, 2200, (128, 128, 2, False)), (1300, 4104, (128, 128, 2, False)),
    (200, 648, (64, 64, 4, False)), (2100, 1000, (64, 64, 4, False)),
    (200, 136, (32, 64, 4, False)), (1300, 136, (32, 64, 4, False)),
    (2100, 4104, (256, 256, 4, False)), (2500, 4240, (256, 256, 4, False)),
]
LINEAR = [(d, *c) for d in ("bf16", "fp16") for c in TILES_16] + [("fp32", *c) for c in TILES_32]

# sizes of the types, K, N, the tile, rows named by index arrays
LONG = [4500, 31, 0, 1, 33, 64, 500, 95, 1000, 0, 257, 32, 700, 5, 63, 128]
MANY = [3, 0, 70, 1, 33] * 80
CUT = [150000, 3, 0, 100004]
WGRAD_16 = [
    (LONG, 1032, 1048, (256, 256, 4, False), False), (LONG, 1032, 1048, (128, 128, 2, False), True),
    (LONG, 1027, 1041, (128, 128, 2, True), False), (LONG, 1027, 1041, (128, 128, 2, True), True),
    ([20000], 520, 264, (128, 128, 2, False), False), ([3, 20000, 0, 700], 333, 301, (128, 128, 2, True), False),
    (MANY, 136, 64, (128, 64, 2, False), False), (MANY, 64, 136, (64, 128, 2, False), True),
    (MANY, 133, 61, (128, 64, 2, True), True), (MANY, 61, 133, (64, 128, 2, True), False),
    (CUT, 128, 64, (64, 64, 2, False), True), (CUT, 136, 64, (128, 64, 2, False), True), (CUT, 64, 136, (64, 128, 2, False), False),
    (LONG, 64, 72, (64, 64, 2, False), False), (LONG, 61, 72, (64, 64, 2, True), True),
]
WGRAD_32 = [
    (LONG, 132, 260, (64, 64, 2, False), False), (LONG, 131, 257, (64, 64, 2, True), True), (CUT, 64, 72, (64, 64, 2, False), True),
]
WGRAD = [(d, *c) for d in ("bf16", "fp16") for c in WGRAD_16] + [("fp32", *c) for c in WGRAD_32]

CODE = {"fp32": 0, "bf16": 1, "fp16": 2, "fp8": 3}
ADDRESS = 0x10000     # looked at as an address only


def select(dtype, rows, num_types, K, N, trans=0, gather=None, x_rows=None, ldx=None, X=ADDRESS, W=ADDRESS):
    import ctypes
    from paper_2301_06284_amd import rgnn
    t = rgnn.Tile()
    st = rgnn.lib().rgnn_typed_linear_select_tile(CODE[dtype], X, rows if x_rows is None else x_rows, K if ldx is None else ldx,
                                                  gather, num_types, rows, W, K, N, trans, ctypes.byref(t))
    return (t.rows, t.cols, t.stages, bool(t.any)) if st == 0 else st


def select_wgrad(dtype, rows, num_types, K, N, gather=None, ldx=None, X=ADDRESS):
    import ctypes
    from paper_2301_06284_amd import rgnn
    t = rgnn.Tile()
    st = rgnn.lib().rgnn_typed_linear_wgrad_select_tile(CODE[dtype], X, rows, K if ldx is None else ldx, gather, ADDRESS, rows, N, None,
                                                        num_types, rows, K, N, ctypes.byref(t))
    return (t.rows, t.cols, t.stages, bool(t.any)) if st == 0 else st


# ------------------------------------------------------------------ the choice, on the CPU

@pytest.mark.parametrize("dtype,K,N,tile", LINEAR)
@pytest.mark.parametrize("trans", [0, 1])
def test_tile_of_linear(dtype, K, N, tile, trans):
    assert select(dtype, M, T, K, N, trans) == tile


@pytest.mark.parametrize("K,N,tile", TILES_8)
def test_tile_of_fp8(K, N, tile):
    assert select("fp8", M, T, K, N, 1, ldx=-(-K // 128) * 128) == tile


@pytest.mark.parametrize("dtype,sizes,K,N,tile,index", WGRAD)
def test_tile_of_wgrad(dtype, sizes, K, N, tile, index):
    assert select_wgrad(dtype, BEFORE + sum(sizes) + BEHIND, len(sizes), K, N, ADDRESS if index else None) == tile


def test_tile_by_address():
    """One operand that is no whole vectors sends the call to the tiles for any address; gathered rows whose offsets
    pass 32 bits do not take the wide tile."""
    wide = (256, 256, 4, False)
    assert select("bf16", 16384, 1, 2048, 4096) == wide
    assert select("bf16", 16384, 1, 2048, 4096, gather=ADDRESS, x_rows=(1 << 20) - 1) == wide
    assert select("bf16", 16384, 1, 2048, 4096, gather=ADDRESS, x_rows=1 << 20) == (128, 128, 2, False)
    assert select("bf16", 16384, 1, 2048, 4096, x_rows=1 << 20) == wide
    for kw in (dict(X=ADDRESS + 2), dict(W=ADDRESS + 8), dict(ldx=2052)):
        assert select("bf16", 16384, 1, 2048, 4096, **kw)[3]
    assert select_wgrad("bf16", 8192, 16, 2048, 1536) == wide
    assert select_wgrad("bf16", 8192, 16, 2048, 1536, ldx=1 << 23) == (128, 128, 2, False)
    assert select_wgrad("bf16", 8192, 16, 2048, 1536, X=ADDRESS + 4) == (128, 128, 2, True)


@pytest.mark.parametrize("rows,num_types,K,N,tile", [
    (292, 1, 1561, 333, (32, 64)), (8192, 1, 2047, 1535, (128, 128)), (16384, 1, 2047, 1535, (128, 128)),
    (5000, 8, 777, 1001, (128, 128)), (2048, 16, 1001, 2001, (128, 128)), (300007, 96, 61, 61, (128, 64)),
])
def test_tile_of_any_address(rows, num_types, K, N, tile):
    """The fastest tile where the others measured a tenth to a half slower."""
    assert select("bf16", rows, num_types, K, N)[:2] == tile


def test_tile_refusals():
    from paper_2301_06284_amd import rgnn
    assert rgnn.lib().rgnn_typed_linear_select_tile(1, ADDRESS, 10, 64, None, 3, 10, ADDRESS, 64, 32, 0, None) == -1
    assert rgnn.lib().rgnn_typed_linear_wgrad_select_tile(1, ADDRESS, 10, 64, None, ADDRESS, 10, 32, None, 3, 10, 64, 32, None) == -1
    assert select("bf16", 10, 0, 64, 32) == -1 and select("bf16", 10, 3, 64, 32, 2) == -1 and select("bf16", 10, 3, 64, 32, -1) == -1
    assert select("fp8", 10, 3, 128, 32, 0) == -1 and select("fp8", 10, 3, 100, 32, 1, ldx=100) == -1
    assert select("bf16", 10, 3, 64, 32, ldx=63) == -1 and select("bf16", 10, 70000, 64, 32) == -2
    assert select("bf16", 10, 3, 64, 32, x_rows=9) == -1 and select_wgrad("bf16", 10, 3, 64, 32, ldx=63) == -1
    assert select_wgrad("fp8", 10, 3, 64, 32) == -1


# ------------------------------------------------------------------ the tiles, on the GPU

def indices(g, rows, count, unnamed):
    """`count` rows that repeat, never `unnamed`, some outside."""
    import torch
    index = torch.randint(0, rows, (count,), generator=g, device="cuda", dtype=torch.int32)
    index[index == unnamed] = unnamed + 1
    index[BEFORE + 3::211], index[BEFORE + 7::307], index[BEFORE + 1::401] = -1, rows, 2 ** 31 - 1
    return index


def places(g, count):
    """A permutation with some places outside."""
    import torch
    index = torch.randperm(count, generator=g, device="cuda").to(torch.int32)
    index[BEFORE + 4::223], index[BEFORE + 9::331] = -1, -2 ** 31
    index[BEFORE + 6::419] = count + 1000
    return index


def check_placed(y, full, ref, size, scatter, n, what, grouped=0.0):
    """y, a part of `full` that held 7 everywhere: the owned positions' rows at their places, 7 in all others."""
    import torch
    own = torch.arange(PTR[0], PTR[-1], device="cuda")
    at = own if scatter is None else scatter[own].long()
    inside = (at >= 0) & (at < y.shape[0])
    own, at = own[inside], at[inside]
    got, ref, size = y[at], ref[own], size[own]
    if y.dtype == torch.float16:
        # rounding takes 65520 (half a step above the largest, 65504) and more to infinity: results that
        # are off by less than `off` must be infinite above 65520 + off, finite below 65520 - off
        off, over = (n * 2.0 ** -23 + grouped) * size, torch.isinf(got)
        assert (ref.abs() >= 65520 - off)[over].all() and (got.sign() == ref.sign())[over].all(), what
        assert over[ref.abs() > 65520 + off].all(), what
        got, ref, size = (t.masked_fill(over, 0.0) for t in (got, ref, size))
    close(got, ref, size, n, what, grouped)
    rest = torch.ones(full.shape, dtype=torch.bool, device="cuda")
    first = (full.shape[1] - y.shape[1]) // 2
    rest[at, first:first + y.shape[1]] = False
    assert (full[rest] == 7.0).all(), f"{what}: written elsewhere"


@gpu
@pytest.mark.parametrize("dtype,K,N,tile", LINEAR)
@pytest.mark.parametrize("trans", [False, True])
def test_linear(dtype, K, N, tile, trans):
    import torch
    from paper_2301_06284_amd import rgnn
    dt = types()[dtype]
    g = torch.Generator(device="cuda").manual_seed(K + N + trans)
    dptr = torch.tensor(PTR, dtype=torch.int64, device="cuda")
    pad = 3 if tile[3] else 8
    w = (torch.randn(T, K, N, generator=g, device="cuda") / math.sqrt(K)).to(dt)
    w[2] = float("nan")                                   # the type without rows
    wk = w.transpose(1, 2).contiguous() if trans else w
    for indexed in (False, True):
        rows = 700 if indexed else M
        wide = torch.full((rows, K + pad), float("nan"), dtype=dt, device="cuda")
        x = wide[:, :K]
        x.copy_((torch.randn(rows, K, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(dt))
        x[640, K // 2] = float("nan")                     # spoils its own outputs, no others
        gather = scatter = None
        if indexed:
            x[17] = float("nan")
            gather, scatter = indices(g, rows, M, 17), places(g, M)
        else:
            x[:PTR[0]], x[PTR[-1]:] = float("nan"), float("nan")
        assert rgnn.typed_linear_select_tile(x, wk, gather, scatter, trans) == tile
        ref, size = linear_ref(x, PTR, w, gather, M)
        size = torch.nan_to_num(size)
        for yt in {dt, torch.float32}:
            full = torch.full((M, N + 2 * pad), 7.0, dtype=yt, device="cuda")
            print(f"tile {tile} {dtype} trans={trans} {K}x{N} indexed={indexed} {yt}", flush=True)
            rgnn.typed_linear(x, dptr, wk, full[:, pad:pad + N], gather=gather, scatter=scatter, trans_w=trans)
            check_placed(full[:, pad:pad + N], full, ref, size, scatter, K, f"indexed={indexed} {yt}")


def integers(g, shape, most, dt):
    import torch
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda", dtype=torch.int32).to(dt)


@gpu
@pytest.mark.parametrize("dtype,K,N,tile", LINEAR)
@pytest.mark.parametrize("trans", [False, True])
def test_linear_exact(dtype, K, N, tile, trans):
    """Integers of -4 .. 4: sums below 2^15, exact in fp32, rounded once in 16 bits."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt = types()[dtype]
    g = torch.Generator(device="cuda").manual_seed(K * N + trans)
    dptr = torch.tensor(PTR, dtype=torch.int64, device="cuda")
    x, w = integers(g, (700, K), 4, dt), integers(g, (T, K, N), 4, dt)
    gather, scatter = indices(g, 700, M, 17), torch.randperm(M, generator=g, device="cuda").to(torch.int32)
    wk = w.transpose(1, 2).contiguous() if trans else w
    assert rgnn.typed_linear_select_tile(x, wk, gather, scatter, trans) == tile
    ref, _ = linear_ref(x, PTR, w, gather, M)
    for yt in {dt, torch.float32}:
        y = torch.full((M, N), float("nan"), dtype=yt, device="cuda")
        print(f"tile {tile} exact {dtype} trans={trans} {K}x{N} {yt}", flush=True)
        rgnn.typed_linear(x, dptr, wk, y, gather=gather, scatter=scatter, trans_w=trans)
        assert torch.equal(y[scatter.long()][PTR[0]:PTR[-1]], ref[PTR[0]:PTR[-1]].to(yt))


@gpu
@pytest.mark.parametrize("out", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("K,N,tile", TILES_8)
def test_fp8_linear(K, N, tile, out):
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(K + N)
    dptr = torch.tensor(PTR, dtype=torch.int64, device="cuda")
    w = torch.randn(T, K, N, generator=g, device="cuda") / math.sqrt(K)
    w[0, :max(1, K // 2)] *= 300                          # blocks of very different scale
    w[3, :, N // 2:] /= 1000
    w[2] = float("nan")
    wq, ws = rgnn.fp8_quantize_weights(w)
    wv = fp8_values(wq, ws, 128).transpose(1, 2)
    for indexed in (False, True):
        rows = 700 if indexed else M
        x = torch.randn(rows, K, generator=g, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda"))
        x[640, K // 2] = float("nan")
        gather = scatter = None
        if indexed:
            x[17] = float("nan")
            gather, scatter = indices(g, rows, M, 17), places(g, M)
        xq, xs = rgnn.fp8_quantize_rows(x)
        assert rgnn.typed_linear_select_tile(xq, wq, gather, scatter) == tile
        ref, size = linear_ref(fp8_values(xq, xs, 1), PTR, wv, gather, M)
        full = torch.full((M, N + 16), 7.0, dtype=types()[out], device="cuda")
        print(f"tile {tile} fp8 {K}x{N} indexed={indexed} {out}", flush=True)
        rgnn.typed_linear_fp8(xq, xs, dptr, wq, ws, full[:, 8:8 + N], gather=gather, scatter=scatter)
        check_placed(full[:, 8:8 + N], full, ref, torch.nan_to_num(size), scatter, K, f"indexed={indexed} {out}", GROUPED)


@gpu
@pytest.mark.parametrize("K,N,tile", TILES_8)
def test_fp8_linear_exact(K, N, tile):
    """Codes of -4 .. 4 under scales of 1/2, 1 and 2: every product and sum is a multiple of 1/4 below
    2^18, whose bits all fit, so that the fp32 result is exact."""
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(K)
    Kp, Ks = rgnn.fp8_widths(K)
    codes = lambda *s: torch.randint(-4, 5, s, generator=g, device="cuda").float()  # noqa: E731
    scales = lambda *s: torch.randint(126, 129, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    xq, wq = codes(M, Kp), codes(T, N, Kp)
    xq[:, K:], wq[:, :, K:] = 0, 0
    xq, wq = xq.to(torch.float8_e4m3fn), wq.to(torch.float8_e4m3fn)
    xs, ws = scales(M, Ks), scales(T, -(-N // 128), Ks)
    assert rgnn.typed_linear_select_tile(xq, wq) == tile
    ref, _ = linear_ref(fp8_values(xq, xs, 1), PTR, fp8_values(wq, ws, 128).transpose(1, 2), None, M)
    y = torch.full((M, N), float("nan"), device="cuda")
    print(f"tile {tile} fp8 exact {K}x{N}", flush=True)
    rgnn.typed_linear_fp8(xq, xs, torch.tensor(PTR, device="cuda"), wq, ws, y)
    assert torch.equal(y[PTR[0]:PTR[-1]].double(), ref[PTR[0]:PTR[-1]])


@gpu
@pytest.mark.parametrize("dtype,sizes,K,N,tile,index", WGRAD)
def test_wgrad(dtype, sizes, K, N, tile, index):
    import torch
    from paper_2301_06284_amd import rgnn
    dt, num = types()[dtype], len(sizes)
    ptr = [BEFORE] + (BEFORE + np.cumsum(sizes)).tolist()
    count = ptr[-1] + BEHIND
    g = torch.Generator(device="cuda").manual_seed(K + N + index)
    rows = 3000 if index else count
    pad = 3 if tile[3] else 8

    def matrix(width):
        full = torch.full((rows, width + pad), float("nan"), dtype=dt, device="cuda")
        full[:, :width] = torch.randn(rows, width, generator=g, device="cuda").to(dt)
        return full[:, :width]

    x, dy = matrix(K), matrix(N)
    gather = dyg = None
    if index:
        x[17], dy[29] = float("nan"), float("nan")
        gather, dyg = indices(g, rows, count, 17), indices(g, rows, count, 29)
        gather[BEFORE + 11::503], dyg[BEFORE + 11::503] = 17, -1           # NaN beside a row outside
        gather[BEFORE + 13::509], dyg[BEFORE + 13::509] = rows + 5, 29
    else:
        for m in (x, dy):
            m[:ptr[0]], m[ptr[-1]:] = float("nan"), float("nan")
    assert rgnn.typed_linear_wgrad_select_tile(x, dy, num, gather, dyg) == tile
    dptr = torch.tensor(ptr, dtype=torch.int64, device="cuda")
    if index:
        # a position outside either matrix adds nothing: the reference takes both rows as zeros
        out = (gather < 0) | (gather >= rows) | (dyg < 0) | (dyg >= rows)
        a, b = (torch.where(out, torch.full_like(i, -1), i) for i in (gather, dyg))
        xr, dyr = torch.nan_to_num(x), torch.nan_to_num(dy)
    else:
        a = b = None
        xr, dyr = x, dy
    ref, size = wgrad_ref(xr, dyr, ptr, a, b, num)
    for wt in {dt, torch.float32}:
        results = []
        for _ in range(2):
            dw = torch.full((num, K, N), float("nan"), dtype=wt, device="cuda")
            print(f"tile {tile} wgrad {dtype} {K}x{N} index={index} {wt}", flush=True)
            rgnn.typed_linear_wgrad(x, dy, dptr, dw, workspace(dt, count, num, K, N), gather=gather, dy_gather=dyg)
            results.append(dw)
        close(results[0], ref, size, max(sizes), f"{wt}")
        assert torch.equal(*results)
        assert all((results[0][t] == 0).all() for t in range(num) if sizes[t] == 0)


@gpu
@pytest.mark.parametrize("dtype,sizes,K,N,tile,index", WGRAD)
def test_wgrad_exact(dtype, sizes, K, N, tile, index):
    """Integers of -3 .. 3: sums of 150 000 products stay below 2^24, exact in fp32, rounded once in 16 bits."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, num = types()[dtype], len(sizes)
    ptr = [BEFORE] + (BEFORE + np.cumsum(sizes)).tolist()
    count = ptr[-1] + BEHIND
    g = torch.Generator(device="cuda").manual_seed(K * N + index)
    rows = 3000 if index else count
    x, dy = integers(g, (rows, K), 3, dt), integers(g, (rows, N), 3, dt)
    gather, dyg = (torch.randint(0, rows, (count,), generator=g, device="cuda", dtype=torch.int32) if index else None for _ in range(2))
    assert rgnn.typed_linear_wgrad_select_tile(x, dy, num, gather, dyg) == tile
    dptr = torch.tensor(ptr, dtype=torch.int64, device="cuda")
    ref, _ = wgrad_ref(x, dy, ptr, gather, dyg, num)
    for wt in {dt, torch.float32}:
        dw = torch.full((num, K, N), float("nan"), dtype=wt, device="cuda")
        print(f"tile {tile} wgrad exact {dtype} {K}x{N} index={index} {wt}", flush=True)
        rgnn.typed_linear_wgrad(x, dy, dptr, dw, workspace(dt, count, num, K, N), gather=gather, dy_gather=dyg)
        assert torch.equal(dw, ref.to(wt))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_wide_rows_near_and_beyond_32_bits(dtype):
    """Gathered rows whose byte offsets lie just below 2^32 (the wide tile) and beyond (another one), and positions
    far into a matrix that is not gathered (the wide tile), against 64 bits."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, K, N, count = types()[dtype], 2048, 4096, 16384
    g = torch.Generator(device="cuda").manual_seed(9)
    tail = torch.randn(1000, K, generator=g, device="cuda").to(dt)
    w = (torch.randn(2, K, N, generator=g, device="cuda") / 45).to(dt)
    index = torch.randint(0, 1000, (count,), generator=g, device="cuda", dtype=torch.int32)
    ptr = [0, 7001, count]
    ref, size = linear_ref(tail, ptr, w, index, count)
    first, first_size = linear_ref(tail, [0, 300, 1000], w, None, 1000)
    for rows, tile in (((1 << 20) - 1, (256, 256, 4, False)), ((1 << 20) + 700, (128, 128, 2, False))):   # 4096 bytes each
        x = torch.zeros(rows, K, dtype=dt, device="cuda")
        x[-1000:] = tail
        gather = index + (rows - 1000)
        assert rgnn.typed_linear_select_tile(x, w, gather) == tile
        y = torch.full((count, N), float("nan"), dtype=dt, device="cuda")
        print(f"{rows} rows {dtype}", flush=True)
        rgnn.typed_linear(x, torch.tensor(ptr, device="cuda"), w, y, gather=gather)
        close(y, ref, size, K, f"{rows} rows")
        at = rows - 1000
        scatter = torch.arange(-at, rows - at, dtype=torch.int32, device="cuda")
        assert rgnn.typed_linear_select_tile(x, w, None, scatter) == (256, 256, 4, False)
        z = torch.full((1000, N), float("nan"), dtype=dt, device="cuda")
        rgnn.typed_linear(x, torch.tensor([at, at + 300, rows], device="cuda"), w, z, scatter=scatter)
        close(z, first, first_size, K, f"far in {rows} rows")
        del x, y, z
