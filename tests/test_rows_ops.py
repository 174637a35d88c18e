"""The norm with residual, dropout and 8-bit outputs, its gradients, dropout, and the typed linear in 8-bit integers on
the GPU, against plain 64-bit implementations.

Tolerances, with u = 2^-24 (half a step of fp32) and h half a step of the output's type (eps / 2), each relative to the
value that is rounded; sums over a row are kept in 64 bits and add nothing that counts:
  sum     one rounding to fp32 (the product is not rounded before the addition) and one to its type: u + h.
  rstd    formed in 64 bits, rounded once: u.
  y       from sum and rstd as they were given out: (r s) w, two products: 2 u + h.
  codes   the values of y in fp32, whose two products torch forms alike, so codes and scales are equal bit for bit.
  dr      s (g - n c) + dsum with n = r s, g = dY w, c = mean(g n).  n, g: u each; a product g n: 3 u, so c is off by
          3 u A + u |c|, A = mean |g n|; n c is off by |n| 3 u A + 3 u |n c| (n, c, the product); the difference's
          rounding u (|g| + |n c|), g's own u |g|; the product with s u of itself; the sum with dsum u of itself.
          Together u (s (3 |g| + 5 |n c| + 3 |n| A) + |dr| + |dsum|) + h.
  dx      dr times the factor: u more.
  dW      a sum of `rows` products dY n with u (n) and u (product or fused sum) each, rows + 34 additions of u of the
          sum of magnitudes: (rows + 36) u sum |dY n| + h.
Second orders are covered by a factor 1 + 2^-10."""
import math

import numpy as np
import pytest

from rows_reference import keep, numbers

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SECOND = 1 + 2.0 ** -10
HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # eps / 2
LEAST = {"fp32": 2.0 ** -150, "bf16": 2.0 ** -134, "fp16": 2.0 ** -25}  # half the least subnormal


@pytest.fixture(scope="module", autouse=True)
def gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2301_06284_amd import rgnn  # noqa: F401  (fails loudly if not built)
    torch.cuda.set_device(0)


def types():
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def name_of(dtype):
    return {v: k for k, v in types().items()}[dtype]


def close(got, ref, off, what):
    """|got - ref| at most `off` (before the last rounding) and the rounding to got's type."""
    import torch
    t = name_of(got.dtype)
    tol = SECOND * (off + HALF[t] * (ref.abs() + off)) + LEAST[t]
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN in other places"
    over = ((got.double() - ref).abs() / tol).masked_fill(nan, 0.0)
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the tolerance"


def matrix(g, rows, cols, dtype, pad=0, shift=0):
    """Rows of different size inside a wider matrix of NaN, from element `shift` of it on."""
    import torch
    wide = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    m = wide[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_((torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(dtype))
    return m


def like(m, dtype=None, fill=7.0):
    """A matrix of m's strides, with a margin that must stay as it is."""
    import torch
    rows, cols = m.shape
    ld = max(m.stride(0), cols)
    wide = torch.full((rows * ld + 16,), fill, dtype=dtype or m.dtype, device="cuda")
    return wide[8:8 + rows * ld].view(rows, ld)[:, :cols], wide


def margin_kept(m, wide, fill=7.0):
    """Nothing of the buffer but the matrix was written."""
    import torch
    mask = torch.ones_like(wide, dtype=torch.bool)
    rows, cols = m.shape
    ld = m.stride(0) if rows > 1 else max(m.stride(0), cols)
    mask[8:8 + rows * ld].view(rows, ld)[:, :cols] = False
    assert (wide[mask] == fill).all(), "written outside the matrix"


def rng_of(seed, offset):
    import torch
    return torch.tensor([seed, offset], dtype=torch.int64, device="cuda")


def factor(p):
    return float(np.float32(1.0 / (1.0 - p))) if p < 1 else 0.0


def kept(rows, cols, p, seed, offset, call):
    import torch
    return torch.from_numpy(keep(rows, cols, p, seed % 2 ** 64, offset, call)).cuda()


SEED, OFFSET, CALL = -1234567890123456789, 2 ** 40 + 77, 5


def check_norm(rows, cols, x_t, res_t, w_t, y_t, p=0.0, pad=0, shift=0, eps=1e-6, keep_sum=True, seed=0, in_place=False):
    """One call against the definition, in all its outputs."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"norm {rows}x{cols} x={x_t} res={res_t} w={w_t} y={y_t} p={p} pad={pad} shift={shift}", flush=True)
    T = types()
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + cols)
    x = matrix(g, rows, cols, T[x_t], pad, shift)
    if rows > 2:
        x[1] = 0
    res = matrix(g, rows, cols, T[res_t], pad, shift) if res_t else None
    if res is not None and rows > 2:
        res[1] = 0
    w = (1 + torch.randn(cols, generator=g, device="cuda") * 0.3).to(T[w_t]) if w_t else None
    drop = rgnn.Dropout(p, rng_of(SEED, OFFSET), CALL) if p is not None and p > 0 else None
    sum_t = T[res_t or x_t]
    total, wide_sum = like(x, sum_t) if keep_sum else (None, None)
    rstd = torch.full((rows,), 7.0, device="cuda")
    eight = y_t in ("e4m3", "int8")
    scales = None
    if y_t == "e4m3":
        kp, ks = rgnn.fp8_widths(cols)
        y = torch.empty(rows, kp, dtype=torch.uint8, device="cuda").fill_(0x55).view(torch.float8_e4m3fn)
        scales = torch.full((rows, ks), 7, dtype=torch.uint8, device="cuda")
    elif y_t == "int8":
        y = torch.full((rows, rgnn.fp8_widths(cols)[0]), 7, dtype=torch.int8, device="cuda")
        scales = torch.full((rows,), 7.0, device="cuda")
    else:
        y, wide_y = like(x, T[y_t])
    x0 = x.clone()
    res0 = None if res is None else res.clone()
    if in_place:
        total, y = res, x
    rgnn.rms_norm(x, w, y, eps=eps, residual=res, sum=total, scales=scales, rstd=rstd, dropout=drop)
    torch.cuda.synchronize()
    # the sum, from the definition
    r = x0.double()
    if drop is not None:
        r = torch.where(kept(rows, cols, p, SEED, OFFSET, CALL), r * factor(p), torch.zeros_like(r))
    if res0 is not None:
        r = r + res0.double()
    if total is not None:
        close(total, r, U * r.abs(), "sum")
        r = total.double()
        if not in_place:
            margin_kept(total, wide_sum)
    else:
        r = r.float().to(sum_t).double()
    s = 1 / torch.sqrt(r.square().mean(dim=1) + eps)
    assert ((rstd.double() - s).abs() <= SECOND * U * s + 2.0 ** -150).all(), "rstd"
    weight = torch.ones(cols, device="cuda") if w is None else w.float()
    if not eight:
        ref = r * rstd.double()[:, None] * weight.double()
        close(y, ref, 2 * U * ref.abs() + 2.0 ** -148, "y")
        if not in_place:
            margin_kept(y, wide_y)
        return
    y32 = r.float() * rstd[:, None] * weight
    check_codes(y32, y, scales, y_t)


def check_codes(y32, codes, scales, kind):
    """Codes and scales of fp32 values, bit for bit."""
    import torch
    rows, cols = y32.shape
    kp = codes.shape[1]
    if kind == "e4m3":
        b = torch.nn.functional.pad(y32, (0, kp - cols)).view(rows, -1, 128)
        bits = b.abs().amax(dim=2).view(torch.int32)
        e = (((bits + 0x1FFFFF) >> 23) - 8).clamp(1, 254)
        ref = (b * torch.exp2((127 - e).float()).unsqueeze(2)).view(rows, kp).to(torch.float8_e4m3fn)
        want = torch.full((rows, scales.shape[1]), 127, dtype=torch.int32, device="cuda")
        want[:, :e.shape[1]] = e
        assert torch.equal(scales.int(), want), "scale bytes"
        assert torch.equal(codes.view(torch.uint8) & 0x7F, ref.view(torch.uint8) & 0x7F), "codes"
        assert torch.equal(codes.float(), ref.float())
    else:
        scale = (y32.abs().amax(dim=1).double() / 127.0).float().clamp(min=2.0 ** -126)      # the quotient rounded once
        ref = torch.round(y32.double() * (1.0 / scale).double()[:, None]).to(torch.int8)
        assert torch.equal(scales, scale), "scales"
        assert torch.equal(codes[:, :cols], ref), "codes"
        assert (codes[:, cols:] == 0).all()


COLS = [1, 7, 8, 9, 24, 32, 33, 64, 65, 100, 128, 129, 256, 257, 333, 512, 513, 1000, 1025, 2048, 2050, 4096, 4100, 8192, 8200, 16384,
        16400, 32768, 32776, 40001]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("x_t,res_t,w_t,y_t", [("bf16", "bf16", "bf16", "bf16"), ("fp16", "fp32", "fp32", "fp16"),
                                               ("fp32", "fp32", "fp32", "fp32"), ("bf16", "fp32", "bf16", "e4m3"),
                                               ("fp16", "fp16", "fp16", "int8"), ("fp32", "", "", "e4m3"),
                                               ("fp32", "fp32", "fp32", "int8")])
def test_norm(cols, x_t, res_t, w_t, y_t):
    for rows in (1, 37) if cols > 4096 else (1, 3, 300):
        check_norm(rows, cols, x_t, res_t, w_t, y_t)


@pytest.mark.parametrize("cols", [257, 333, 511, 513, 1001, 1023])
@pytest.mark.parametrize("x_t,res_t,w_t,y_t", [("bf16", "bf16", "bf16", "bf16"), ("fp16", "fp32", "fp32", "e4m3"), ("fp32", "fp32", "fp32", "int8")])
def test_norm_of_many_rows_that_end_inside_a_vector(cols, x_t, res_t, w_t, y_t):
    check_norm(4099, cols, x_t, res_t, w_t, y_t, p=0.1 if y_t == "bf16" else 0.0)


@pytest.mark.parametrize("x_t,res_t,w_t,y_t", [("bf16", "", "bf16", "bf16"), ("fp16", "", "", "fp32"), ("fp32", "bf16", "bf16", "bf16"),
                                               ("fp32", "", "fp16", "fp16"), ("bf16", "bf16", "fp32", "fp32"),
                                               ("fp32", "fp16", "fp32", "fp32"), ("bf16", "fp32", "", "fp32"),
                                               ("fp16", "fp16", "fp32", "e4m3"), ("fp32", "bf16", "bf16", "int8")])
@pytest.mark.parametrize("cols", [24, 130, 1536, 5000])
def test_norm_types(cols, x_t, res_t, w_t, y_t):
    check_norm(67, cols, x_t, res_t, w_t, y_t)


@pytest.mark.parametrize("cols,pad,shift", [(64, 8, 8), (100, 3, 1), (333, 0, 0), (333, 1, 5), (2048, 24, 3), (2048, 8, 8), (2047, 2, 2),
                                            (5000, 1, 7), (33000, 9, 1)])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_norm_any_address(kind, cols, pad, shift):
    """Rows of wider matrices of NaN, on any address of an element."""
    check_norm(41, cols, kind, kind, kind, kind, pad=pad, shift=shift)
    check_norm(5, cols, kind, "fp32", kind, "e4m3", pad=pad, shift=shift)
    check_norm(5, cols, kind, kind, kind, "int8", pad=pad, shift=shift)


@pytest.mark.parametrize("cols", [1, 30, 333, 2048, 6000, 16390, 33001])
@pytest.mark.parametrize("p", [0.1, 0.5, 0.999, 1.0])
def test_norm_with_dropout(cols, p):
    check_norm(65 if cols < 4096 else 7, cols, "bf16", "bf16", "bf16", "bf16", p=p)
    check_norm(9, cols, "fp16", "fp32", "fp32", "fp16", p=p)
    check_norm(9, cols, "fp32", "", "fp32", "fp32", p=p)
    check_norm(9, cols, "fp32", "fp32", "fp32", "int8", p=p)


@pytest.mark.parametrize("cols", [64, 333, 2048, 33000])
@pytest.mark.parametrize("y_t", ["bf16", "e4m3", "int8"])
def test_norm_without_a_kept_sum(cols, y_t):
    check_norm(33, cols, "bf16", "bf16", "bf16", y_t, p=0.1, keep_sum=False)


@pytest.mark.parametrize("cols", [100, 1000, 1001, 2048, 8192, 33000])
def test_norm_with_dropout_into_codes(cols):
    check_norm(21, cols, "bf16", "bf16", "bf16", "e4m3", p=0.2)
    check_norm(21, cols, "fp16", "fp32", "fp32", "int8", p=0.2)


@pytest.mark.parametrize("cols", [64, 333, 2048, 33000])
@pytest.mark.parametrize("x_t,sum_t", [("fp32", "bf16"), ("bf16", "fp32"), ("fp32", "fp16")])
def test_norm_keeps_the_sum_in_another_type(cols, x_t, sum_t):
    """Without a residual the sum may be of any type; y is of what is kept."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"sum of another type {cols} {x_t} {sum_t}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = matrix(g, 19, cols, types()[x_t])
    total, rstd = torch.empty(19, cols, dtype=types()[sum_t], device="cuda"), torch.empty(19, device="cuda")
    y = torch.empty(19, cols, device="cuda")
    rgnn.rms_norm(x, None, y, sum=total, rstd=rstd)
    assert torch.equal(total, x.to(types()[sum_t]))
    s = 1 / torch.sqrt(total.double().square().mean(dim=1) + 1e-6)
    assert ((rstd.double() - s).abs() <= SECOND * U * s).all()
    ref = total.double() * rstd.double()[:, None]
    close(y, ref, 2 * U * ref.abs() + 2.0 ** -148, "y")


def test_two_graphs_share_a_workspace():
    """Two captured backward passes with one workspace, replayed in turn with eager work in between."""
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(6)
    sets, graphs, wanted = [], [], []
    ws = torch.empty(rgnn.rms_norm_backward_workspace_size(5000, 512), dtype=torch.uint8, device="cuda")
    for rows, cols in ((5000, 512), (700, 100)):
        x, dy = matrix(g, rows, cols, torch.float32), matrix(g, rows, cols, torch.float32)
        sets.append((dy, x, torch.ones(rows, device="cuda"), torch.ones(cols, device="cuda"), torch.empty_like(x), torch.empty(cols, device="cuda")))
    for dy, x, rstd, w, dx, dw in sets:
        work = lambda: rgnn.rms_norm_backward(dy, x, rstd, w, dX=dx, dW=dw, ws=ws)  # noqa: E731,B023
        work()
        torch.cuda.synchronize()
        wanted.append((dx.clone(), dw.clone()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            work()
        graphs.append(graph)
    for turn in range(3):
        for (dy, x, rstd, w, dx, dw), graph, want in zip(sets, graphs, wanted):
            dx.zero_(), dw.zero_()
            if turn == 1:
                ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])


@pytest.mark.parametrize("cols", [64, 100, 2048, 33000])
def test_norm_in_place(cols):
    """The sum over the residual, the output over x."""
    for p in (0.0, 0.3):
        check_norm(33, cols, "fp16", "fp16", "fp32", "fp16", p=p, in_place=True)


@pytest.mark.parametrize("cols", [40, 128, 1000, 4096, 33000])
@pytest.mark.parametrize("y_t", ["fp32", "e4m3", "int8"])
def test_norm_of_rows_that_are_not_finite(cols, y_t):
    """Zeros, infinities and NaN spoil their own rows alone; huge and tiny rows have finite norms."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"norm of rows that are not finite {cols} {y_t}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(12, cols, generator=g, device="cuda")
    x[1] = 0
    x[3, cols // 2] = float("inf")
    x[5, cols - 1] = float("nan")
    x[7] *= 1e38 / x[7].abs().max()
    x[9] *= 1e-30
    ref = x.double()
    kp, ks = rgnn.fp8_widths(cols)
    y, scales = {"fp32": (torch.empty_like(x), None),
                 "e4m3": (torch.empty(12, kp, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(12, ks, dtype=torch.uint8, device="cuda")),
                 "int8": (torch.empty(12, kp, dtype=torch.int8, device="cuda"), torch.empty(12, device="cuda"))}[y_t]
    rstd = torch.empty(12, device="cuda")
    eps = 0.0 if y_t == "fp32" else 1e-60
    rgnn.rms_norm(x, None, y, eps=eps, scales=scales, rstd=rstd)
    good = [0, 2, 4, 6, 7, 8, 9, 10, 11]
    # rstd of the row of 1e-30 is 1e30, of that of 1e38 about 1e-38: both normal numbers of fp32
    s = 1 / (ref[good].square().mean(dim=1) + eps).sqrt()
    assert ((rstd[good].double() - s).abs() <= SECOND * U * s).all()
    y32 = x * rstd[:, None]
    if y_t == "fp32":
        want = ref[good] * rstd[good].double()[:, None]
        close(y[good], want, 2 * U * want.abs() + 2.0 ** -148, "y")
        assert torch.isnan(y[1]).all()               # 0 / 0 without eps
        assert torch.isnan(y[5]).all() and torch.isnan(y[3, cols // 2])
        assert cols == 1 or (y[3, :cols // 2] == 0).all()
    elif y_t == "int8":
        check_codes(y32[good], y[good], scales[good], "int8")
        assert (y[1] == 0).all() and scales[1] == 2.0 ** -126
        assert torch.isnan(scales[[3, 5]]).all() and (y[[3, 5]] == 0).all()
    else:
        check_codes(y32[good], y[good], scales[good], "e4m3")
        assert (y[1].float() == 0).all() and (scales[1, :kp // 128] == 1).all()
        assert (scales[5, :kp // 128] == 255).all() and torch.isnan(y[5].float()).all()
        assert scales[3, cols // 2 // 128] == 255


def test_codes_are_those_of_the_quantisers():
    """Straight into 8 bits: the same codes and scales as by way of fp32 rows."""
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(3)
    for rows, cols in ((1, 64), (300, 100), (77, 1536), (19, 5000), (3, 33000)):
        print(f"codes {rows}x{cols}", flush=True)
        x, res = matrix(g, rows, cols, torch.bfloat16), matrix(g, rows, cols, torch.bfloat16)
        w = torch.randn(cols, generator=g, device="cuda").bfloat16()
        y = torch.empty(rows, cols, device="cuda")
        rgnn.rms_norm(x, w, y, residual=res)
        kp, ks = rgnn.fp8_widths(cols)
        c, s = torch.empty(rows, kp, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(rows, ks, dtype=torch.uint8, device="cuda")
        rgnn.rms_norm(x, w, c, residual=res, scales=s)
        c2, s2 = rgnn.fp8_quantize_rows(y)
        assert torch.equal(c.view(torch.uint8), c2.view(torch.uint8)) and torch.equal(s, s2)
        c, s = torch.empty(rows, kp, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        rgnn.rms_norm(x, w, c, residual=res, scales=s)
        c2, s2 = rgnn.int8_quantize_rows(y)
        assert torch.equal(c, c2) and torch.equal(s, s2)


# ------------------------------------------------------------------ gradients

def backward_ref(dy, r, rstd, w, dsum):
    """(dr, its error bound, dW, its sum of magnitudes) in 64 bits from what the call was given."""
    import torch
    dy, r, s = dy.double(), r.double(), rstd.double()[:, None]
    w = torch.ones(r.shape[1], dtype=torch.float64, device="cuda") if w is None else w.double()
    n, gr = r * s, dy * w
    c, size = (gr * n).mean(dim=1, keepdim=True), (gr * n).abs().mean(dim=1, keepdim=True)
    dr = s * (gr - n * c)
    d = torch.zeros_like(dr) if dsum is None else dsum.double()
    off = U * (s * (3 * gr.abs() + 5 * (n * c).abs() + 3 * n.abs() * size) + (dr + d).abs() + d.abs())
    return dr + d, off, (dy * n).sum(dim=0), (dy * n).abs().sum(dim=0)


def check_backward(rows, cols, dy_t, sum_t, w_t, dx_t, dw_t, p=0.0, pad=0, shift=0, with_dsum=True, wanted=("dres", "dx", "dw"),
                   in_place=False, seed=0):
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"norm backward {rows}x{cols} dy={dy_t} sum={sum_t} w={w_t} dx={dx_t} dw={dw_t} p={p} pad={pad} shift={shift} {wanted}", flush=True)
    T = types()
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 5 + cols)
    dy, r = matrix(g, rows, cols, T[dy_t], pad, shift), matrix(g, rows, cols, T[sum_t], pad, shift)
    dsum = matrix(g, rows, cols, T[sum_t], pad, shift) if with_dsum else None
    w = (1 + torch.randn(cols, generator=g, device="cuda") * 0.3).to(T[w_t]) if w_t else None
    rstd = (1 / torch.sqrt(r.double().square().mean(dim=1) + 1e-6)).float()
    drop = rgnn.Dropout(p, rng_of(SEED, OFFSET), CALL) if p else None
    dr, off, dw_ref, dw_size = backward_ref(dy, r, rstd, w, dsum)
    dres, wide_r = like(r) if "dres" in wanted else (None, None)
    dx, wide_x = like(dy, T[dx_t]) if "dx" in wanted else (None, None)
    if in_place:
        dres, dx = dsum, dy
    dw = torch.full((cols,), 7.0, dtype=T[dw_t], device="cuda") if "dw" in wanted else None
    need = rgnn.rms_norm_backward_workspace_size(rows, cols)
    ws = torch.full((need // 4 + 8,), 7.0, device="cuda") if dw is not None else None
    rgnn.rms_norm_backward(dy, r, rstd, w, d_sum=dsum, d_residual=dres, dX=dx, dW=dw, ws=None if ws is None else ws[:need // 4],
                           dropout=drop)
    torch.cuda.synchronize()
    if dres is not None:
        close(dres, dr, off, "d_residual")
        if not in_place:
            margin_kept(dres, wide_r)
    if dx is not None:
        if p:
            k, f = kept(rows, cols, p, SEED, OFFSET, CALL), factor(p)
            zero = torch.zeros_like(dr)
            dr, off = torch.where(k, dr * f, zero), torch.where(k, off * f + U * (dr * f).abs(), zero)
        close(dx, dr, off, "dX")
        if not in_place:
            margin_kept(dx, wide_x)
    if dw is not None:
        close(dw, dw_ref, (rows + 36) * U * dw_size, "dW")
        assert (ws[need // 4:] == 7.0).all(), "written behind the workspace"


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dy_t,sum_t,w_t,dx_t,dw_t", [("bf16", "bf16", "bf16", "bf16", "bf16"), ("fp16", "fp32", "fp32", "fp16", "fp32"),
                                                      ("fp32", "fp32", "fp32", "fp32", "fp32")])
def test_norm_backward(cols, dy_t, sum_t, w_t, dx_t, dw_t):
    for rows in (1, 40) if cols > 4096 else (1, 3, 300):
        check_backward(rows, cols, dy_t, sum_t, w_t, dx_t, dw_t)


@pytest.mark.parametrize("rows,cols", [(2 ** 19 + 3, 5), (2 ** 18 + 77, 8), (2 ** 17 + 9, 24), (5000, 64), (2 ** 16 + 5, 40), (3001, 333), (2100, 2048), (1500, 5000), (300, 12000), (300, 33000)])
def test_norm_backward_many_rows(rows, cols):
    """More rows than workgroups, so that each takes several."""
    check_backward(rows, cols, "bf16", "bf16", "fp32", "bf16", "fp32", p=0.1)


@pytest.mark.parametrize("dy_t,sum_t,w_t,dx_t,dw_t", [("fp32", "bf16", "bf16", "bf16", "fp32"), ("bf16", "fp32", "", "fp32", "bf16"),
                                                      ("fp16", "fp16", "fp32", "fp32", "fp16"), ("fp32", "fp32", "fp16", "fp16", "fp16")])
@pytest.mark.parametrize("cols", [24, 130, 1536, 5000])
def test_norm_backward_types(cols, dy_t, sum_t, w_t, dx_t, dw_t):
    check_backward(67, cols, dy_t, sum_t, w_t, dx_t, dw_t, with_dsum=False)
    check_backward(67, cols, dy_t, sum_t, w_t, dx_t, dw_t, p=0.5)


@pytest.mark.parametrize("wanted", [("dres",), ("dx",), ("dw",), ("dx", "dw"), ("dres", "dx")])
@pytest.mark.parametrize("cols", [64, 2048, 33000])
def test_norm_backward_parts(cols, wanted):
    check_backward(50, cols, "bf16", "bf16", "bf16", "bf16", "bf16", p=0.25, wanted=wanted)


@pytest.mark.parametrize("cols,pad,shift", [(64, 8, 8), (100, 3, 1), (333, 1, 5), (2048, 24, 3), (2047, 2, 2), (5000, 1, 7), (33000, 9, 1)])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_norm_backward_any_address(kind, cols, pad, shift):
    check_backward(41, cols, kind, kind, kind, kind, kind, pad=pad, shift=shift, p=0.1)


@pytest.mark.parametrize("cols", [64, 2048, 33000])
def test_norm_backward_in_place(cols):
    check_backward(50, cols, "fp16", "fp16", "fp32", "fp16", "fp32", p=0.25, in_place=True)


def test_norm_backward_without_rows():
    import torch
    from paper_2301_06284_amd import rgnn
    dw = torch.full((333,), 7.0, device="cuda")
    e = torch.empty(0, 333, device="cuda")
    rgnn.rms_norm_backward(e, e, torch.empty(0, device="cuda"), torch.ones(333, device="cuda"), dX=e, dW=dw)
    rgnn.rms_norm(e, torch.ones(333, device="cuda"), e)
    rgnn.dropout(e, e, rgnn.Dropout(0.5, rng_of(1, 2)))
    assert (dw == 0).all()


@pytest.mark.parametrize("cols", [40, 333, 2048])
def test_norm_gradients_against_differences(cols):
    """L = sum(y G) + sum(r H), along a random direction of (x, residual, w): the kernels' own difference quotient.
    Its truncation is that of the 64-bit formula with the same step, evaluated here.  Noise, which the quotient divides by
    2 step: x, residual and the sum are rounded, so that r is off by at most d = 2 u (f |x| + |residual|), which reaches L through
    H and through dy/dr, s (|g| + |n| A) at most; y is off by 4 u |y| more (w, rstd, two products).  And the gradients' own bounds."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"differences {cols}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    rows, p, step, eps = 23, 0.3, 2.0 ** -6, 1e-3
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, res, w = randn(rows, cols), randn(rows, cols), 1 + 0.3 * randn(cols)
    vx, vr, vw = randn(rows, cols), randn(rows, cols), randn(cols)
    G, H = randn(rows, cols), randn(rows, cols)
    drop = rgnn.Dropout(p, rng_of(SEED, OFFSET), CALL)
    k = kept(rows, cols, p, SEED, OFFSET, CALL)

    def loss64(t):
        xt, rt, wt = x.double() + t * vx.double(), res.double() + t * vr.double(), w.double() + t * vw.double()
        r = rt + torch.where(k, xt * factor(p), torch.zeros_like(xt))
        y = r / torch.sqrt(r.square().mean(dim=1, keepdim=True) + eps) * wt
        return float((y * G).sum() + (r * H).sum())

    def loss(t):
        y, r = torch.empty_like(x), torch.empty_like(x)
        rgnn.rms_norm(x + t * vx, w + t * vw, y, eps=eps, residual=res + t * vr, sum=r, dropout=drop)
        d = 2 * U * ((x + t * vx).abs() * factor(p) + (res + t * vr).abs()).double()
        gw, inv = (G * (w + t * vw)).double(), 1 / torch.sqrt(r.double().square().mean(dim=1, keepdim=True) + eps)
        n = r.double() * inv
        slope = inv * (gw.abs() + n.abs() * (gw * n).abs().mean(dim=1, keepdim=True))
        noise = SECOND * float((d * (H.abs() + slope)).sum() + 4 * U * (y * G).double().abs().sum())
        return float((y.double() * G.double()).sum() + (r.double() * H.double()).sum()), noise
    y, r, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    rgnn.rms_norm(x, w, y, eps=eps, residual=res, sum=r, rstd=rstd, dropout=drop)
    dx, dres, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(rgnn.rms_norm_backward_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
    rgnn.rms_norm_backward(G, r, rstd, w, d_sum=H, d_residual=dres, dX=dx, dW=dw, ws=ws, dropout=drop)
    along = float((dx.double() * vx.double()).sum() + (dres.double() * vr.double()).sum() + (dw.double() * vw.double()).sum())
    a, na = loss(step)
    b, nb = loss(-step)
    quotient = (a - b) / (2 * step)
    truncation = abs((loss64(step) - loss64(-step)) / (2 * step) - (loss64(2.0 ** -12) - loss64(-2.0 ** -12)) / 2.0 ** -11)
    _, off, _, size = backward_ref(G, r, rstd, w, H)
    off = off + U * dres.double().abs()
    own = float((off * (vr.abs() + 2 * factor(p) * vx.abs())).sum() + (rows + 37) * U * (size * vw.abs()).sum())
    tol = 1.01 * truncation + (na + nb) / (2 * step) + SECOND * own
    assert abs(quotient - along) <= tol, (quotient, along, tol)
    assert tol < 0.05 * max(abs(along), math.sqrt(rows * cols))     # the bound says something


# ------------------------------------------------------------------ dropout

def check_dropout(rows, cols, x_t, y_t, with_res, p, pad=0, shift=0, in_place=None, seed=SEED, offset=OFFSET, call=CALL):
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"dropout {rows}x{cols} x={x_t} y={y_t} res={with_res} p={p} pad={pad} shift={shift} {in_place}", flush=True)
    T = types()
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = matrix(g, rows, cols, T[x_t], pad, shift)
    res = matrix(g, rows, cols, T[y_t], pad, shift) if with_res else None
    y, wide = (x, None) if in_place == "x" else (res, None) if in_place == "res" else like(x, T[y_t])
    ref = torch.where(kept(rows, cols, p, seed, offset, call), x.double() * factor(p), torch.zeros(1, dtype=torch.float64, device="cuda"))
    if with_res:
        ref = ref + res.double()
    rgnn.dropout(x, y, rgnn.Dropout(p, rng_of(seed, offset), call), residual=res)
    torch.cuda.synchronize()
    close(y, ref, U * ref.abs(), "dropout")
    if not with_res and p < 1:
        zero = x.double() * factor(p) == 0
        assert torch.equal((y == 0) | zero, (ref == 0) | zero)
    if wide is not None:
        margin_kept(y, wide)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 3), (5, 7), (300, 8), (292, 64), (1000, 77), (129, 100), (17, 2048), (3, 8192), (2, 8200),
                                       (5, 20001), (4099, 333), (70000, 5)])
@pytest.mark.parametrize("x_t,y_t,with_res", [("bf16", "bf16", True), ("fp16", "fp16", False), ("fp32", "fp32", True), ("fp32", "bf16", False),
                                              ("fp16", "fp32", True)])
def test_dropout(rows, cols, x_t, y_t, with_res):
    check_dropout(rows, cols, x_t, y_t, with_res, 0.1)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -33, 2.0 ** -32, 0.3, 0.5, 1 - 2.0 ** -20, 1.0])
def test_dropout_probabilities(p):
    for with_res in (False, True):
        check_dropout(203, 333, "fp32", "fp32", with_res, p)
        check_dropout(203, 333, "bf16", "bf16", with_res, p)


@pytest.mark.parametrize("cols,pad,shift", [(64, 8, 8), (77, 24, 0), (100, 3, 1), (333, 1, 5), (2048, 24, 3)])
@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp32"])
def test_dropout_any_address(kind, cols, pad, shift):
    check_dropout(101, cols, kind, kind, True, 0.5, pad=pad, shift=shift)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_dropout_in_place(kind):
    check_dropout(205, 333, kind, kind, False, 0.4, in_place="x")
    check_dropout(205, 333, kind, kind, True, 0.4, in_place="res")
    check_dropout(205, 333, kind, kind, True, 0.4, in_place="x")


@pytest.mark.parametrize("seed,offset,call", [(0, 0, 0), (-1, -1, 0), (-1, -1, 1), (2 ** 63 - 1, 2 ** 63 - 1, 1), (5, 2 ** 32 - 1, 1), (5, 7, -8)])
def test_dropout_seeds_and_offsets(seed, offset, call):
    """Whole 64-bit seeds and offsets; the offset's sum with the call wraps."""
    check_dropout(33, 100, "fp32", "fp32", False, 0.5, seed=seed, offset=offset, call=call)


def test_dropped_values_are_zero_whatever_they_were():
    import torch
    from paper_2301_06284_amd import rgnn
    x = torch.full((64, 200), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = torch.empty_like(x)
    rgnn.dropout(x, y, rgnn.Dropout(0.5, rng_of(SEED, OFFSET), CALL))
    k = kept(64, 200, 0.5, SEED, OFFSET, CALL)
    assert (y[~k] == 0).all() and not torch.isfinite(y[k]).any()
    res = torch.ones_like(x)
    rgnn.dropout(x, y, rgnn.Dropout(0.5, rng_of(SEED, OFFSET), CALL), residual=res)
    assert (y[~k] == 1).all()


def test_dropout_share():
    """The share of dropped values, within 6 standard deviations, and the masks of two calls, rows and seeds are apart."""
    import torch
    from paper_2301_06284_amd import rgnn
    x = torch.ones(4096, 1024, device="cuda")
    n, masks = x.numel(), []
    for p, call, seed in ((0.1, 0, 1), (0.1, 1, 1), (0.1, 0, 2), (0.7, 0, 1)):
        y = torch.empty_like(x)
        rgnn.dropout(x, y, rgnn.Dropout(p, rng_of(seed, 9), call))
        gone = y == 0
        assert abs(float(gone.double().mean()) - p) <= 6 * math.sqrt(p * (1 - p) / n)
        masks.append(gone)
    for a, b in ((0, 1), (0, 2), (1, 2)):
        both = float((masks[a] & masks[b]).double().mean())
        assert abs(both - 0.01) <= 6 * math.sqrt(0.01 * 0.99 / n)
    near = float((masks[0][1:] & masks[0][:-1]).double().mean())
    assert abs(near - 0.01) <= 6 * math.sqrt(2 * 0.01 * 0.99 / n)
    assert (masks[0] <= masks[3]).all()          # one number for all probabilities


def test_dropout_moves_with_the_generator_in_a_graph():
    """A captured forward and backward pass: each replay drops by the offset that the device holds then; the program's own
    work runs in between."""
    import torch
    from paper_2301_06284_amd import rgnn
    rows, cols, p = 77, 333, 0.4
    g = torch.Generator(device="cuda").manual_seed(1)
    x, res, w = matrix(g, rows, cols, torch.float32), matrix(g, rows, cols, torch.float32), torch.ones(cols, device="cuda")
    rng = rng_of(SEED, 100)
    drop, drop2 = rgnn.Dropout(p, rng, 0), rgnn.Dropout(p, rng, 1)
    y, r, rstd, z = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty_like(x)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(rgnn.rms_norm_backward_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")

    def work():
        rgnn.rms_norm(x, w, y, residual=res, sum=r, rstd=rstd, dropout=drop)
        rgnn.dropout(y, z, drop2)
        rgnn.rms_norm_backward(z, r, rstd, w, dX=dx, dW=dw, ws=ws, dropout=drop)
        rng[1].add_(2)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for turn in range(4):
        rng.copy_(rng_of(SEED, 1000 + turn))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, r, z, dx, dw)]
        assert int(rng[1]) == 1002 + turn
        rng.copy_(rng_of(SEED, 1000 + turn))
        work()
        torch.cuda.synchronize()
        for a, b in zip(got, (y, r, z, dx, dw)):
            assert torch.equal(a, b)
        assert torch.equal(z == 0, ~kept(rows, cols, p, SEED, 1000 + turn, 1) | (y == 0))
        for t in (y, r, z, dx, dw):
            t.fill_(float("nan"))


# ------------------------------------------------------------------ 8-bit integers

@pytest.mark.parametrize("K", [1, 8, 100, 128, 129, 500, 1000, 2048, 2050, 4096, 8000, 16384, 16500, 40001])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_int8_rows(dtype, K):
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"int8 rows {dtype} {K}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(K)
    for rows, pad, shift in ((1, 0, 0), (70, 0, 0), (33, 3, 1), (33, 8, 8)):
        x = matrix(g, rows, K, types()[dtype], pad, shift)
        if rows > 20:
            x[3] = 0
            x[7, K // 2] = float("inf")
            x[9, K - 1] = float("nan")
            if dtype == "fp32":
                x[11] *= 1e-42 / x[11].abs().max()        # subnormal
                x[13] *= 3e38 / x[13].abs().max()
        buffer = torch.full((rows * rgnn.fp8_widths(K)[0] + 16,), 7, dtype=torch.int8, device="cuda")
        codes, scales = rgnn.int8_quantize_rows(x, codes=buffer[:-16].view(rows, -1))
        finite = torch.isfinite(x).all(dim=1)            # (a factor above overflows where a row's largest is below 1)
        good = finite.nonzero().view(-1)
        check_codes(x[good].float(), codes[good], scales[good], "int8")
        assert (buffer[-16:] == 7).all()
        if rows > 20:
            assert not finite[7] and not finite[9] and finite.sum() >= rows - 3
            assert torch.isnan(scales[~finite]).all() and (codes[~finite] == 0).all()
            assert scales[3] == 2.0 ** -126


@pytest.mark.parametrize("K,N", [(1, 1), (8, 8), (100, 77), (64, 64), (128, 65), (130, 63), (500, 128), (2048, 136), (1000, 1), (1030, 40), (2049, 33), (4096, 72), (4100, 72)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_int8_weights(dtype, K, N):
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"int8 weights {dtype} {K}x{N}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(K + N)
    w = (torch.randn(3, K, N, generator=g, device="cuda") * torch.exp(torch.randn(3, 1, N, generator=g, device="cuda"))).to(types()[dtype])
    w[1, :, N // 2] = 0
    w[2, K // 2, N - 1] = float("nan")
    w[0, K - 1, 0] = float("-inf")
    codes, scales = rgnn.int8_quantize_weights(w)
    bad = torch.isnan(scales)
    want = torch.zeros_like(bad)
    want[2, N - 1] = want[0, 0] = True
    assert torch.equal(bad, want) and (codes[bad] == 0).all()
    flat = w.float().transpose(1, 2)
    check_codes(flat[~bad], codes[~bad], scales[~bad], "int8")


PTRS = {"ragged": [0, 5, 5, 200, 201, 777, 1000], "one": [0, 1], "few": [3, 3, 4, 4, 20, 37, 37], "dense": [0, 515]}


def int8_case(ptr, K, N, seed=0, extra=0, rows=None):
    """Codes over their whole range, -128 among them, zero behind K, and scales."""
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(seed)
    kp, M, T = rgnn.fp8_widths(K)[0], ptr[-1] + extra, len(ptr) - 1
    rows = rows or M
    x = torch.randint(-128, 128, (rows, kp), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (T, N, kp), generator=g, device="cuda", dtype=torch.int8)
    x[:, K:], w[:, :, K:] = 0, 0
    xs = torch.exp(torch.randn(rows, generator=g, device="cuda"))
    ws = torch.exp(torch.randn(T, N, generator=g, device="cuda"))
    return g, x, xs, w, ws, torch.tensor(ptr, dtype=torch.int64, device="cuda")


def int8_ref(x, xs, w, ws, ptr, gather, M):
    """The definition, bit for bit: exact sums in 64 bits (whole numbers below 2^53), then fp32."""
    import torch
    pos = torch.arange(M, device="cuda") if gather is None else gather.long()
    ok = (pos >= 0) & (pos < x.shape[0])
    at = pos.clamp(0, x.shape[0] - 1)
    y = torch.zeros(M, w.shape[1], device="cuda")
    for t in range(w.shape[0]):
        a, b = ptr[t], ptr[t + 1]
        if b > a:
            total = x[at[a:b]].double() @ w[t].double().t()
            y[a:b] = total.float() * xs[at[a:b], None] * ws[t]
    return torch.where(ok[:, None], y, torch.zeros_like(y))


@pytest.mark.parametrize("K,N", [(1, 1), (8, 8), (64, 64), (100, 77), (128, 130), (264, 136), (513, 320), (1024, 64), (2050, 129)])
@pytest.mark.parametrize("shape", list(PTRS))
@pytest.mark.parametrize("out", ["fp32", "bf16", "fp16"])
def test_int8_linear(K, N, shape, out):
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"int8 linear {K}x{N} {shape} {out}", flush=True)
    ptr = PTRS[shape]
    _, x, xs, w, ws, dptr = int8_case(ptr, K, N, K + N, extra=30)
    if out == "fp16":      # inside fp16's range
        ws *= 1e-4
    M = x.shape[0]
    y = torch.full((M, N), 7.0, dtype=types()[out], device="cuda")
    rgnn.typed_linear_int8(x, xs, dptr, w, ws, y)
    ref = int8_ref(x, xs, w, ws, ptr, None, M).to(types()[out])
    own = slice(ptr[0], ptr[-1])
    assert torch.equal(y[own], ref[own])
    assert (torch.cat([y[:ptr[0]], y[ptr[-1]:]]) == 7.0).all()


# sizes that take each of the tiles
TILES = [(16, 4, 512, 320, (32, 64, 4)), (300, 8, 2050, 1001, (32, 64, 4)), (3000, 3, 256, 320, (64, 64, 4)), (40, 3, 100, 500, (128, 64, 1)),
         (5000, 40, 128, 64, (128, 64, 1)), (300, 30, 100, 2048, (128, 128, 1)), (2000, 3, 256, 1024, (128, 64, 2)),
         (2000, 30, 256, 2045, (128, 128, 2)), (9000, 30, 1024, 768, (128, 128, 2)), (8192, 1, 1024, 4096, (256, 256, 4)),
         (16000, 3, 1010, 1023, (256, 256, 4))]


@pytest.mark.parametrize("rows,T,K,N,tile", TILES)
def test_int8_linear_tiles(rows, T, K, N, tile):
    """Each tile, with gathered and scattered rows, some outside, NaN scales where nothing may be read; the row and the output of a
    NaN scale."""
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(rows)
    cut = torch.sort(torch.randint(0, rows + 1, (T - 1,), generator=g, device="cuda")).values.tolist()
    ptr = [0] + cut + [rows]
    _, x, xs, w, ws, dptr = int8_case(ptr, K, N, rows + K, rows=max(20, rows // 2))
    gather = torch.randint(0, x.shape[0], (rows,), generator=g, device="cuda", dtype=torch.int32)
    gather[gather == 17] = 18
    xs[17] = float("nan")
    gather[3::211], gather[7::307], gather[1::401] = -1, x.shape[0], 2 ** 31 - 1
    scatter = torch.randperm(rows, generator=g, device="cuda").to(torch.int32)
    lost = scatter[4::97].clone()
    scatter[4::97] = -1
    take = rgnn.typed_linear_select_tile(x, w, gather=gather, scatter=scatter)
    print(f"int8 tile {rows} rows of {T} types {K}x{N}: {take}", flush=True)
    assert take[:3] == tile
    for nan in (False, True):
        if nan:
            xs[int(gather[5])] = float("nan")
            ws[-1, N - 1] = float("nan")
        y = torch.full((rows, N + 5), 7.0, dtype=torch.bfloat16, device="cuda")
        rgnn.typed_linear_int8(x, xs, dptr, w, ws, y[:, :N], gather=gather, scatter=scatter)
        ref = int8_ref(x, xs, w, ws, ptr, gather, rows).bfloat16()
        want = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
        ok = scatter >= 0
        want[scatter[ok].long()] = ref[ok]
        assert torch.equal(torch.isnan(want), torch.isnan(y[:, :N]))
        assert torch.equal(torch.nan_to_num(want.float()), torch.nan_to_num(y[:, :N].float()))
        assert (y[:, N:] == 7.0).all() and (y[lost.long()] == 7.0).all()


def test_int8_linear_largest_sums():
    """The longest k, with the codes of largest magnitude: sums next to 2^31."""
    import torch
    from paper_2301_06284_amd import rgnn
    K = 130944
    for rows, N in ((3, 8), (300, 256)):
        print(f"int8 largest sums {rows} {N}", flush=True)
        x = torch.full((rows, K), -128, dtype=torch.int8, device="cuda")
        w = torch.full((1, N, K), -128, dtype=torch.int8, device="cuda")
        x[1] = 127
        y = torch.empty(rows, N, device="cuda")
        rgnn.typed_linear_int8(x, torch.ones(rows, device="cuda"), torch.tensor([0, rows], device="cuda"), w, torch.ones(1, N, device="cuda"), y)
        assert (y[0] == float(np.float32(K * 16384))).all() and (y[1] == float(np.float32(-K * 16256))).all()


def test_int8_linear_of_no_rows():
    import torch
    from paper_2301_06284_amd import rgnn
    _, x, xs, w, ws, dptr = int8_case([0, 4, 9], 64, 32)
    gather = torch.full((9,), -1, dtype=torch.int32, device="cuda")
    y = torch.full((9, 32), 7.0, device="cuda")
    rgnn.typed_linear_int8(x[:0], xs[:0], dptr, w, ws, y, gather=gather)
    assert (y == 0).all()
    rgnn.typed_linear_int8(x[:0], xs[:0], dptr, w, ws, y[:0])


# ------------------------------------------------------------------ large matrices, streams, together

def test_rows_beyond_32_bits():
    """Matrices whose last rows lie beyond 2^32 bytes and 2^31 elements."""
    import torch
    from paper_2301_06284_amd import rgnn
    rows, cols, ld = 33000, 72, 70000
    print("rows beyond 32 bits", flush=True)
    big = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    x, y = big.view(rows, ld)[:, 8:8 + cols], out.view(rows, ld)[:, 8:8 + cols]
    g = torch.Generator(device="cuda").manual_seed(2)
    x.copy_(torch.randn(rows, cols, generator=g, device="cuda"))
    w, small = torch.ones(cols, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    drop = rgnn.Dropout(0.5, rng_of(1, 2))
    xc = x.contiguous()
    rgnn.rms_norm(x, w, y)
    rgnn.rms_norm(xc, w, small)
    assert torch.equal(y, small)
    rgnn.dropout(x, y, drop)
    rgnn.dropout(xc, small, drop)
    assert torch.equal(y, small)
    a, b = rgnn.int8_quantize_rows(x), rgnn.int8_quantize_rows(xc)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    rstd = torch.ones(rows, device="cuda")
    rgnn.rms_norm_backward(x, x, rstd, w, dX=y)
    rgnn.rms_norm_backward(xc, xc, rstd, w, dX=small)
    assert torch.equal(y, small)


def test_more_workgroups_than_a_launch_is_wide():
    """2^22 rows and more of 1024 threads each, which along one axis were 2^32 threads.  All rows repeat the first 64."""
    import torch
    from paper_2301_06284_amd import rgnn
    rows, cols = 2 ** 22 + 64, 4104
    print("more workgroups than a launch is wide", flush=True)
    first = matrix(torch.Generator(device="cuda").manual_seed(6), 64, cols, torch.bfloat16)
    w, small = torch.ones(cols, dtype=torch.bfloat16, device="cuda"), torch.empty_like(first)
    x = first.repeat(rows // 64, 1)
    rgnn.rms_norm(first, w, small)
    rgnn.rms_norm(x, w, x)
    for part in x.view(-1, 64, cols).split(4096):
        assert (part == small).all()
    del x, part
    torch.cuda.empty_cache()


def test_streams():
    """Two calls at once on two streams, with workspaces of their own; outputs made in the stream's memory."""
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(4)
    rows, cols = 3000, 1000
    x, dy = matrix(g, rows, cols, torch.float32), matrix(g, rows, cols, torch.float32)
    w = torch.ones(cols, device="cuda")
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            y, rstd, dx, dw = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(w)
            ws = torch.empty(rgnn.rms_norm_backward_workspace_size(rows, cols), dtype=torch.uint8, device="cuda")
        for _ in range(5):
            rgnn.rms_norm(x, w, y, rstd=rstd, stream=s)
            rgnn.rms_norm_backward(dy, x, rstd, w, dX=dx, dW=dw, ws=ws, stream=s)
            codes, scales = rgnn.int8_quantize_rows(y, stream=s)
            rgnn.dropout(dx, dx, rgnn.Dropout(0.0, rng_of(1, 1)), stream=s)
        got.append((y, rstd, dx, dw, codes, scales, ws))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert a.dtype == torch.uint8 or torch.equal(a, b)
    with pytest.raises(ValueError):
        rgnn.int8_quantize_rows(x.cpu())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_train_a_layer(dtype):
    """A residual block as a program runs it, forward and backward: norm of (residual + dropout), typed linear, dropout with the
    residual's addition; its gradients against autograd in 64 bits on the values as they were rounded between the calls.

    Tolerance: the block's outputs pass through the roundings of a chain of at most five tensors of type t, each
    relative to a value that the next call's condition (at most a few units here: rows are normalised) hands on; the norms of the
    differences are held to 8 half steps of t (16-bit) and, in fp32, to K 2^-23 for the products' sums of K summands."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"train a layer {dtype}", flush=True)
    dt, ptr, K, p, eps = types()[dtype], [0, 100, 100, 357, 400], 136, 0.2, 1e-5
    g = torch.Generator(device="cuda").manual_seed(9)
    rows, T = ptr[-1], len(ptr) - 1
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, res = randn(rows, K).to(dt), randn(rows, K).to(dt)
    w, W = (1 + 0.2 * randn(K)).to(dt), (randn(T, K, K) / math.sqrt(K)).to(dt)
    grad = randn(rows, K).to(dt)
    dptr, rng = torch.tensor(ptr, device="cuda"), rng_of(SEED, 3)
    d0, d1 = rgnn.Dropout(p, rng, 0), rgnn.Dropout(p, rng, 1)
    new = lambda t: torch.empty_like(t)  # noqa: E731
    total, y, rstd, z, out = new(x), new(x), torch.empty(rows, device="cuda"), new(x), new(x)
    rgnn.rms_norm(x, w, y, eps=eps, residual=res, sum=total, rstd=rstd, dropout=d0)
    rgnn.typed_linear(y, dptr, W, z)
    rgnn.dropout(z, out, d1, residual=total)
    dz, dy, dx, dres, dw, dW = new(x), new(x), new(x), new(x), new(w), new(W)
    rgnn.dropout(grad, dz, d1)
    rgnn.typed_linear(dz, dptr, W, dy, trans_w=True)
    ws = torch.empty(rgnn.typed_linear_wgrad_workspace_size(dt, rows, T, K, K), dtype=torch.uint8, device="cuda")
    rgnn.typed_linear_wgrad(y, dz, dptr, dW, ws)
    ws = torch.empty(rgnn.rms_norm_backward_workspace_size(rows, K), dtype=torch.uint8, device="cuda")
    rgnn.rms_norm_backward(dy, total, rstd, w, d_sum=grad, d_residual=dres, dX=dx, dW=dw, ws=ws, dropout=d0)
    # the same in 64 bits on the CPU
    leaf = [t.double().cpu().requires_grad_() for t in (x, res, w, W)]
    X, R, V, WW = leaf
    k0, k1 = (torch.from_numpy(keep(rows, K, p, SEED % 2 ** 64, 3, c)) for c in (0, 1))
    zero, f = torch.zeros((), dtype=torch.float64), factor(p)
    S = R + torch.where(k0, X * f, zero)
    Y = S / torch.sqrt(S.square().mean(dim=1, keepdim=True) + eps) * V
    Z = torch.cat([Y[a:b] @ WW[t] for t, (a, b) in enumerate(zip(ptr, ptr[1:]))])
    O = S + torch.where(k1, Z * f, zero)
    O.backward(grad.double().cpu())
    bound = 8 * HALF[dtype] if dtype != "fp32" else K * 2.0 ** -23
    for name, got, ref in (("out", out, O.detach()), ("dx", dx, X.grad), ("dres", dres, R.grad), ("dw", dw, V.grad), ("dW", dW, WW.grad)):
        off = float((got.double().cpu() - ref).norm() / ref.norm())
        assert off <= bound, (name, off, bound)


@pytest.mark.parametrize("rows", [1, 8, 300])
def test_serve_a_layer(rows):
    """Norm into 8 bits and the product that reads them, both forms, against the product of the rows in 64 bits.

    Tolerance of the norm of the difference: int8 codes are off by half a unit of top / 127 at most in rows and in weights, which on
    normal data (top at least 2.5, at most 5.5 standard deviations for these widths) is below 5.5 / 127 / 2 of a standard deviation each;
    e4m3 by 2^-4 each."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"serve a layer {rows}", flush=True)
    T, K, N = 4, 512, 384
    g = torch.Generator(device="cuda").manual_seed(rows)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, res, w = randn(rows, K).bfloat16(), randn(rows, K).bfloat16(), (1 + 0.1 * randn(K)).bfloat16()
    W = (randn(T, K, N) / math.sqrt(K)).bfloat16()
    ptr = [0, rows // 3, rows // 2, rows, rows]
    dptr = torch.tensor(ptr, device="cuda")
    scatter = torch.randperm(rows, generator=g, device="cuda").to(torch.int32)
    total = torch.empty_like(x)
    kp, ks = rgnn.fp8_widths(K)
    r = (x.float() + res.float()).bfloat16().double()
    ref = r / torch.sqrt(r.square().mean(dim=1, keepdim=True) + 1e-6) * w.double()
    ref = torch.cat([ref[a:b] @ W[t].double() for t, (a, b) in enumerate(zip(ptr, ptr[1:]))])
    want = torch.empty_like(ref)
    want[scatter.long()] = ref
    for kind in ("int8", "e4m3"):
        y = torch.empty(rows, N, dtype=torch.bfloat16, device="cuda")
        if kind == "int8":
            wq, ws = rgnn.int8_quantize_weights(W)
            q, s = torch.empty(rows, kp, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
        else:
            wq, ws = rgnn.fp8_quantize_weights(W)
            q, s = torch.empty(rows, kp, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(rows, ks, dtype=torch.uint8, device="cuda")
        call = lambda: (rgnn.rms_norm(x, w, q, residual=res, sum=total, scales=s),  # noqa: E731
                        (rgnn.typed_linear_int8 if kind == "int8" else rgnn.typed_linear_fp8)(q, s, dptr, wq, ws, y, scatter=scatter))
        call()
        off = float((y.double() - want).norm() / want.norm())
        assert off <= (2 * 5.5 / 254 if kind == "int8" else 2 * 2.0 ** -4) + HALF["bf16"], (kind, off)
        first = y.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(3):
            y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, first)


def test_numbers_of_the_generator():
    """The numbers themselves, to 16 bits: thresholds at multiples of 2^-16 bracket each."""
    import torch
    from paper_2301_06284_amd import rgnn
    rows, cols = 9, 37
    want = torch.from_numpy((numbers(rows, cols, 123456789012345, 42) >> np.uint64(16)).astype(np.int64)).cuda()
    low = torch.zeros(rows, cols, dtype=torch.int64, device="cuda")
    x, y = torch.ones(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
    found = torch.zeros_like(low)
    for bit in range(15, -1, -1):      # bit by bit, the elements that share a threshold together
        for t in torch.unique(found + (1 << bit)).tolist():
            rgnn.dropout(x, y, rgnn.Dropout(t / 65536, rng_of(123456789012345, 42)))
            found = torch.where((y != 0) & (found + (1 << bit) == t), found + (1 << bit), found)
    assert torch.equal(found, want)
