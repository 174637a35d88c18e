"""What the norm makes of sums at their ends: rows of zeros under the least eps."""
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
