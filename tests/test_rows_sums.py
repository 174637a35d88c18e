"""What the norm and its gradients make of sums at their ends: rows of zeros under the least eps, and the
weight's gradient over as many rows as give every workgroup several turns, where whole numbers make it exact."""
import pytest

pytestmark = pytest.mark.gpu

MOST = float.fromhex("0x1.fffffep+127")      # the largest fp32 number


@pytest.fixture(scope="module", autouse=True)
def gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2301_06284_amd import rgnn  # noqa: F401  (fails loudly if not built)
    torch.cuda.set_device(0)


@pytest.mark.parametrize("eps", [1e-70, 1e-78, 1e-80, 1e-300, 5e-324])
@pytest.mark.parametrize("cols", [5, 40, 333, 4096, 33000])
@pytest.mark.parametrize("y_t", ["fp32", "bf16", "e4m3", "int8"])
def test_rows_of_zeros_are_zeros_for_any_eps(cols, y_t, eps):
    """1 / sqrt(eps) leaves fp32 for eps below 2^-256 and counts as the largest number there, which makes a row of zeros
    zeros; so does that of rows next to nothing."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"zeros {cols} {y_t} {eps}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn(6, cols, generator=g, device="cuda")
    x[1] = 0
    x[3] = 2.0 ** -140                  # 1 / rms is 2^140
    x[4] = 0
    kp, ks = rgnn.fp8_widths(cols)
    y, scales = {"fp32": (torch.empty_like(x), None), "bf16": (torch.empty_like(x, dtype=torch.bfloat16), None),
                 "e4m3": (torch.empty(6, kp, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(6, ks, dtype=torch.uint8, device="cuda")),
                 "int8": (torch.empty(6, kp, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda"))}[y_t]
    rstd = torch.empty(6, device="cuda")
    rgnn.rms_norm(x, None, y, eps=eps, scales=scales, rstd=rstd)
    s = (1 / torch.sqrt(x.double().square().mean(dim=1) + eps)).clamp(max=MOST)
    assert ((rstd.double() - s).abs() <= (1 + 2.0 ** -10) * 2.0 ** -24 * s).all()
    assert (y[[1, 4]].float() == 0).all()
    if y_t == "e4m3":
        assert (scales[[1, 4], :kp // 128] == 1).all()
    elif y_t == "int8":
        assert (scales[[1, 4]] == 2.0 ** -126).all()
    else:
        assert torch.equal(y, (x * rstd[:, None]).to(y.dtype))      # one rounding each, as the kernel's


def test_rows_of_zeros_without_eps_are_nan():
    import torch
    from paper_2301_06284_amd import rgnn
    x = torch.zeros(2, 64, device="cuda")
    x[1] = 1
    y, rstd = torch.empty_like(x), torch.empty(2, device="cuda")
    rgnn.rms_norm(x, None, y, eps=0.0, rstd=rstd)
    assert torch.isnan(y[0]).all() and rstd[0] == float("inf") and (y[1] == 1).all()


# rows, columns: for each number of lanes and vectors that a row has, more rows than 1024 workgroups (512 beyond 2048
# columns, 256 beyond 4096) take in one turn
TURNS = [(2 ** 19 + 3, 5), (2 ** 18 + 77, 8), (2 ** 17 + 9, 24), (2 ** 17 + 9, 31), (2 ** 16 + 5, 64), (2 ** 16 + 5, 45), (40000, 128),
         (40000, 100), (20001, 256), (20001, 200), (9002, 512), (9002, 333), (9002, 1024), (9002, 1001), (2500, 2048), (2500, 1500),
         (1500, 4096), (1500, 2050), (700, 8192), (700, 5003), (700, 16384), (700, 10001), (700, 20000), (700, 17003), (600, 33000)]


@pytest.mark.parametrize("p", [0.0, 0.25])
@pytest.mark.parametrize("dy_t,sum_t", [("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("rows,cols", TURNS)
def test_weight_gradient_over_several_turns(rows, cols, dy_t, sum_t, p):
    """dY and the sum are whole numbers up to 3 and 1 / rms is 1: products up to 9 and all their sums, below 9 * 2^19 + 27 <
    2^23, are whole numbers that fp32 holds, so dW is exact in any order.  Every turn's share of it is not zero."""
    import torch
    from paper_2301_06284_amd import rgnn
    print(f"dW {rows}x{cols} {dy_t} {sum_t} p={p}", flush=True)
    T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    whole = lambda: torch.randint(-3, 4, (rows, cols), generator=g, device="cuda")  # noqa: E731
    dy, r = whole(), whole()
    want = (dy * r).sum(dim=0)
    groups = rgnn.rms_norm_backward_workspace_size(rows, cols) // (4 * cols)
    lanes = 1 if cols <= 8 else 4 if cols <= 32 else 8 if cols <= 64 else 16 if cols <= 128 else 32 if cols <= 256 else 64 if cols <= 1024 else 256
    turn = groups * (256 // lanes)
    assert rows > turn
    for first in range(0, rows, turn):
        assert (dy[first:first + turn] * r[first:first + turn]).sum(dim=0).any()
    dy, r = dy.to(T[dy_t]), r.to(T[sum_t])
    w, rstd = torch.ones(cols, device="cuda"), torch.ones(rows, device="cuda")
    dw, dx = torch.full((cols,), 7.0, device="cuda"), torch.empty_like(dy)
    ws = torch.full((groups * cols,), 7.0, device="cuda")
    drop = rgnn.Dropout(p, torch.tensor([3, 4], dtype=torch.int64, device="cuda")) if p else None
    rgnn.rms_norm_backward(dy, r, rstd, w, dX=dx, dW=dw, ws=ws, dropout=drop)
    assert torch.equal(dw, want.float())
