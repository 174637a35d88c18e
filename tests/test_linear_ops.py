"""The typed linear over device offsets (forward, input gradient, weight gradient, 8-bit
form) and the AdamW step on the GPU, against plain 64-bit implementations.

Tolerances.  A sum of n products has an error of at most n 2^-23 sum |x w|: products of
16-bit and 8-bit values are exact in fp32, an fp32 product is off by 2^-24 of itself, and
each addition by at most 2^-23 of the partial sum (a matrix core may truncate where it
aligns the summands).  Rounding the result adds half a step of its type: eps / 2 of the
value, or half the least subnormal."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2301_06284_amd import rgnn  # noqa: F401  (fails loudly if not built)
    torch.cuda.set_device(0)


def types():
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


HALF = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # eps / 2
LEAST = {"fp32": 2.0 ** -150, "bf16": 2.0 ** -134, "fp16": 2.0 ** -25}  # half the least subnormal


def name_of(dtype):
    return {v: k for k, v in types().items()}[dtype]


# The 8-bit matrix cores add products in groups of eight, aligned to the group's largest, and
# drop what lies below 2^-13 of its power of two (256 and seven products of 2^-5: exact; seven of
# 2^-6: all dropped; the same for sums of 32 and of 128).  So each of the other seven loses less
# than 2^-13 of the largest product, a group less than 7 * 2^-13 of its largest and so of
# its sum of magnitudes, and a result less than 7 * 2^-13 of `size`.
GROUPED = 7 * 2.0 ** -13


def close(got, ref, size, n, what="", grouped=0.0):
    """got against ref (64 bits), size = the same sum of magnitudes, n summands."""
    import torch
    t = name_of(got.dtype)
    got = got.double()
    off = (n * 2.0 ** -23 + grouped) * size
    tol = off + HALF[t] * (ref.abs() + off) + LEAST[t]
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN in other places"
    over = ((got - ref).abs() / tol).masked_fill(nan, 0.0)
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the tolerance"


def linear_ref(x, ptr, w, gather, M):
    """Rows in position order in 64 bits: (product, product of magnitudes), zero rows where the
    index lies outside X; positions of no type stay None-like (NaN is not used: zero)."""
    import torch
    pos = torch.arange(M, device=x.device) if gather is None else gather.long()
    ok = (pos >= 0) & (pos < x.shape[0])
    rows = x.double()[pos.clamp(0, max(x.shape[0] - 1, 0))]
    rows = torch.where(ok[:, None], rows, torch.zeros_like(rows))
    y = torch.zeros(M, w.shape[2], dtype=torch.float64, device=x.device)
    s = torch.zeros_like(y)
    for t in range(w.shape[0]):
        a, b = ptr[t], ptr[t + 1]
        if b > a:
            y[a:b] = rows[a:b] @ w[t].double()
            s[a:b] = rows[a:b].abs() @ w[t].double().abs()
    return y, s


PTRS = {
    "ragged": [0, 5, 5, 200, 201, 777, 1000],          # empty and one-row types
    "one": [0, 1],
    "few": [3, 3, 4, 4, 20, 37, 37],                   # positions before the first type and behind the last
    "dense": [0, 515],
}


def case(dtype, ptr, K, N, seed=0, extra=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    M, T = ptr[-1] + extra, len(ptr) - 1
    x = (torch.randn(M, K, generator=g, device="cuda") * torch.exp(torch.randn(M, 1, generator=g, device="cuda"))).to(dtype)
    w = (torch.randn(T, K, N, generator=g, device="cuda") / math.sqrt(K)).to(dtype)
    return g, x, w, torch.tensor(ptr, dtype=torch.int64, device="cuda")


WIDTHS = [(1, 1), (8, 8), (16, 24), (64, 64), (64, 128), (128, 64), (77, 100), (100, 77), (160, 8), (264, 136),
          (513, 130), (1024, 320)]


@pytest.mark.parametrize("K,N", WIDTHS)
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", ["ragged", "few"])
def test_linear(dtype, trans, K, N, shape):
    import torch
    from paper_2301_06284_amd import rgnn
    ptr, dt = PTRS[shape], types()[dtype]
    print(f"typed_linear {dtype} trans={trans} {K}x{N} {shape}", flush=True)
    _, x, w, dptr = case(dt, ptr, K, N, K * N + trans, extra=30)
    M = x.shape[0]
    wk = w.transpose(1, 2).contiguous() if trans else w
    for yt in {dt, torch.float32}:
        y = torch.full((M, N), 7.0, dtype=yt, device="cuda")
        rgnn.typed_linear(x, dptr, wk, y, trans_w=trans)
        ref, size = linear_ref(x, ptr, w, None, M)
        own = slice(ptr[0], ptr[-1])
        close(y[own], ref[own], size[own], K, f"{yt}")
        rest = torch.cat([y[:ptr[0]], y[ptr[-1]:]])
        assert (rest == 7.0).all()                       # positions of no type stay as they were


@pytest.mark.parametrize("K,N", [(64, 128), (100, 77), (512, 256), (2048, 136)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_linear_gather_scatter(dtype, K, N):
    """Repeated rows, indices outside the matrix on both sides, rows of a wider matrix, NaN
    wherever nothing may be read."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, ptr = types()[dtype], PTRS["ragged"]
    print(f"gather/scatter {dtype} {K}x{N}", flush=True)
    g, _, w, dptr = case(dt, ptr, K, N, 5)
    M, rows = ptr[-1] + 50, 300
    wide = torch.full((rows, K + 24), float("nan"), dtype=dt, device="cuda")
    x = wide[:, 8:8 + K]
    x.copy_(torch.randn(rows, K, generator=g, device="cuda").to(dt))
    x[17] = float("nan")                                 # a row that no index names
    gather = torch.randint(0, rows, (M,), generator=g, device="cuda", dtype=torch.int32)
    gather[gather == 17] = 18
    gather[3], gather[250], gather[999] = -1, rows, 2 ** 31 - 1
    scatter = torch.randperm(M, generator=g, device="cuda").to(torch.int32)
    scatter[4], scatter[777], scatter[500] = -1, M + 1000, -2 ** 31
    w[1] = float("nan")                                  # the weights of a type without rows
    wide_y = torch.full((M, N + 40), 7.0, dtype=dt, device="cuda")
    y = wide_y[:, 16:16 + N]
    rgnn.typed_linear(x, dptr, w, y, gather=gather, scatter=scatter)
    ref, size = linear_ref(x, ptr, w, gather, M)
    put = torch.zeros(M, dtype=torch.bool, device="cuda")
    for i in range(M):
        j = int(scatter[i])
        if i < ptr[-1] and 0 <= j < M:
            put[j] = True
    pos = torch.arange(ptr[-1], device="cuda")
    pos = pos[(scatter[pos] >= 0) & (scatter[pos] < M)]
    close(y[scatter[pos].long()], ref[pos], size[pos], K)
    assert (y[~put] == 7.0).all()
    assert (wide_y[:, :16] == 7.0).all() and (wide_y[:, 16 + N:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("K,N", [(96, 80), (91, 80)])
def test_linear_nonfinite_rows_stay_apart(dtype, K, N):
    """A row of NaN or infinities spoils its own outputs and no others; NaN in the padding of
    rows, behind the rows and in other types' weights reaches none."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, ptr = types()[dtype], [0, 70, 70, 133]
    g, x, w, dptr = case(dt, ptr, K, N, 9, extra=5)
    wide = torch.full((x.shape[0], 128), float("nan"), dtype=dt, device="cuda")
    wide[:ptr[-1], :K] = x[:ptr[-1]]
    x = wide[:, :K]
    x[12, 3] = float("nan")
    x[100, 0] = float("inf")
    w[1] = float("inf")
    y = torch.zeros(x.shape[0], N, dtype=dt, device="cuda")
    print(f"nonfinite {dtype} {K}x{N}", flush=True)
    rgnn.typed_linear(x, dptr, w, y)
    ref, size = linear_ref(x, ptr, w, None, x.shape[0])
    assert torch.isnan(y[12]).all() and not torch.isfinite(y[100]).any()
    keep = [i for i in range(ptr[-1]) if i not in (12, 100)]
    close(y[keep], ref[keep], size[keep], K)
    assert (y[ptr[-1]:] == 0).all()


@pytest.mark.parametrize("off", [1, 2, 4, 8])
@pytest.mark.parametrize("trans", [False, True])
def test_linear_any_alignment(off, trans):
    """Base addresses and row strides of 2, 4, 8 and 16 bytes."""
    import torch
    from paper_2301_06284_amd import rgnn
    K, N, ptr = 72, 104, PTRS["few"]
    dt = torch.bfloat16
    g, x, w, dptr = case(dt, ptr, K, N, off, extra=3)
    buf = torch.zeros(x.shape[0] * (K + off) + off + 8, dtype=dt, device="cuda")
    xv = buf[off:off + x.shape[0] * (K + off)].view(x.shape[0], K + off)[:, :K]
    xv.copy_(x)
    wk = (w.transpose(1, 2) if trans else w).contiguous()
    wb = torch.zeros(wk.numel() + off, dtype=dt, device="cuda")
    wv = wb[off:].view(wk.shape)
    wv.copy_(wk)
    yb = torch.zeros(x.shape[0] * (N + off) + off + 8, dtype=dt, device="cuda")
    y = yb[off:off + x.shape[0] * (N + off)].view(x.shape[0], N + off)[:, :N]
    print(f"alignment {off} trans={trans}", flush=True)
    rgnn.typed_linear(xv, dptr, wv, y, trans_w=trans)
    ref, size = linear_ref(x, ptr, w, None, x.shape[0])
    close(y[ptr[0]:ptr[-1]], ref[ptr[0]:ptr[-1]], size[ptr[0]:ptr[-1]], K)


def wgrad_ref(x, dy, ptr, gather, dyg, T):
    import torch
    def rows(m, index):
        pos = torch.arange(ptr[-1], device=m.device) if index is None else index[:ptr[-1]].long()
        ok = (pos >= 0) & (pos < m.shape[0])
        r = m.double()[pos.clamp(0, m.shape[0] - 1)]
        return torch.where(ok[:, None], r, torch.zeros_like(r))
    a, b = rows(x, gather), rows(dy, dyg)
    dw = torch.zeros(T, a.shape[1], b.shape[1], dtype=torch.float64, device=x.device)
    size = torch.zeros_like(dw)
    for t in range(T):
        p, q = ptr[t], ptr[t + 1]
        if q > p:
            dw[t] = a[p:q].t() @ b[p:q]
            size[t] = a[p:q].abs().t() @ b[p:q].abs()
    return dw, size


def workspace(dt, M, T, K, N):
    import torch
    from paper_2301_06284_amd import rgnn
    n = rgnn.typed_linear_wgrad_workspace_size(dt, M, T, K, N)
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN: nothing unwritten may be read


@pytest.mark.parametrize("K,N", WIDTHS)
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", ["ragged", "few"])
def test_wgrad(dtype, K, N, shape):
    import torch
    from paper_2301_06284_amd import rgnn
    dt, ptr = types()[dtype], PTRS[shape]
    print(f"wgrad {dtype} {K}x{N} {shape}", flush=True)
    g, x, w, dptr = case(dt, ptr, K, N, 3 * K + N, extra=9)
    M, T = x.shape[0], len(ptr) - 1
    dy = torch.randn(M, N, generator=g, device="cuda").to(dt)
    x[ptr[-1]:], dy[ptr[-1]:] = float("nan"), float("nan")   # behind the last type
    x[:ptr[0]], dy[:ptr[0]] = float("nan"), float("nan")     # before the first one
    ref, size = wgrad_ref(x, dy, ptr, None, None, T)
    rows = max(b - a for a, b in zip(ptr, ptr[1:]))
    for wt in {dt, torch.float32}:
        dw = torch.full((T, K, N), float("nan"), dtype=wt, device="cuda")
        rgnn.typed_linear_wgrad(x, dy, dptr, dw, workspace(dt, M, T, K, N))
        close(dw, ref, size, rows, f"{wt}")


@pytest.mark.parametrize("K,N", [(64, 64), (72, 40), (33, 70), (256, 128), (640, 512)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_wgrad_long_types(dtype, K, N):
    """Types with tens of thousands of rows, whose contraction is split, beside short and empty
    ones; gathered rows that repeat and indices outside; the same bits on a second call."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, ptr = types()[dtype], [0, 30011, 30011, 30012, 33000, 47003]
    T, M, rows = len(ptr) - 1, ptr[-1] + 100, 20000
    g = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn(rows, K, generator=g, device="cuda").to(dt)
    dy = torch.randn(M, N, generator=g, device="cuda").to(dt)
    gather = torch.randint(0, rows, (M,), generator=g, device="cuda", dtype=torch.int32)
    dyg = torch.randperm(M, generator=g, device="cuda").to(torch.int32)
    gather[7], gather[31000], dyg[9], dyg[46000] = -1, rows, -5, M
    dptr = torch.tensor(ptr, dtype=torch.int64, device="cuda")
    print(f"wgrad long {dtype} {K}x{N}", flush=True)
    ref, size = wgrad_ref(x, dy, ptr, gather, dyg, T)
    out = []
    for _ in range(2):
        dw = torch.full((T, K, N), float("nan"), dtype=dt, device="cuda")
        rgnn.typed_linear_wgrad(x, dy, dptr, dw, workspace(dt, M, T, K, N), gather=gather, dy_gather=dyg)
        out.append(dw)
    close(out[0], ref, size, 30011)
    assert torch.equal(out[0], out[1])
    assert (out[0][1] == 0).all()


@pytest.mark.parametrize("T", [1, 255, 256, 257, 700, 3001])
def test_many_types(T):
    """More types than one turn of the offset search covers, most of them empty."""
    import torch
    from paper_2301_06284_amd import rgnn
    rng = np.random.default_rng(T)
    sizes = rng.integers(0, 6, T) * (rng.random(T) < 0.3)
    sizes[rng.integers(0, T)] += 400
    sizes[-1] += 3
    ptr = [0] + np.cumsum(sizes).tolist()
    K, N, dt = 64, 64, torch.bfloat16
    print(f"many types {T}", flush=True)
    g, x, w, dptr = case(dt, ptr, K, N, T)
    M = x.shape[0]
    y = torch.zeros(M, N, dtype=dt, device="cuda")
    rgnn.typed_linear(x, dptr, w, y)
    ref, size = linear_ref(x, ptr, w, None, M)
    close(y, ref, size, K)
    dw = torch.full((T, K, N), float("nan"), dtype=dt, device="cuda")
    rgnn.typed_linear_wgrad(x, y, dptr, dw, workspace(dt, M, T, K, N))
    rw, sw = wgrad_ref(x, y, ptr, None, None, T)
    close(dw, rw, sw, max(sizes))


@pytest.mark.parametrize("M,T,K,N", [(1, 1, 2048, 256), (2, 8, 1024, 512), (16, 8, 1000, 520), (40, 3, 768, 1536),
                                     (130, 4, 512, 2048)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("trans", [False, True])
def test_linear_few_rows(M, T, K, N, dtype, trans):
    """Single tokens: few rows, wide weights."""
    import torch
    from paper_2301_06284_amd import rgnn
    rng = np.random.default_rng(M)
    ptr = [0] + np.cumsum(rng.multinomial(M, np.ones(T) / T)).tolist()
    print(f"few rows {M} {T} {K}x{N} {dtype} {trans}", flush=True)
    g, x, w, dptr = case(types()[dtype], ptr, K, N, M)
    y = torch.full((M, N), float("nan"), dtype=x.dtype, device="cuda")
    rgnn.typed_linear(x, dptr, w.transpose(1, 2).contiguous() if trans else w, y, trans_w=trans)
    ref, size = linear_ref(x, ptr, w, None, M)
    close(y, ref, size, K)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_wide_step(dtype):
    """Full tiles of the widest kernels, ragged at every edge: forward and both gradients."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, ptr, K, N = types()[dtype], [0, 700, 701, 701, 1800, 2405], 1032, 776
    T, M = len(ptr) - 1, ptr[-1] + 11
    g, x, w, dptr = case(dt, ptr, K, N, 1, extra=11)
    dy = torch.randn(M, N, generator=g, device="cuda").to(dt)
    print(f"wide step {dtype}", flush=True)
    y = torch.zeros(M, N, dtype=dt, device="cuda")
    dx = torch.zeros(M, K, dtype=dt, device="cuda")
    dw = torch.zeros(T, K, N, dtype=dt, device="cuda")
    rgnn.typed_linear(x, dptr, w, y)
    rgnn.typed_linear(dy, dptr, w, dx, trans_w=True)
    rgnn.typed_linear_wgrad(x, dy, dptr, dw, workspace(dt, M, T, K, N))
    ref, size = linear_ref(x, ptr, w, None, M)
    close(y, ref, size, K, "y")
    ref, size = linear_ref(dy, ptr, w.transpose(1, 2), None, M)
    close(dx, ref, size, N, "dx")
    ref, size = wgrad_ref(x, dy, ptr, None, None, T)
    close(dw, ref, size, 1099, "dw")


def test_gradients_against_differences():
    """L = sum(Y R): dX and dW in fp32 against central differences of the forward in
    64 bits.  L is linear in X and in W, so the differences are exact but for their rounding."""
    import torch
    from paper_2301_06284_amd import rgnn
    ptr, K, N = [0, 9, 9, 30, 41], 24, 20
    g, x, w, dptr = case(torch.float32, ptr, K, N, 2)
    r = torch.randn(41, N, generator=g, device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    print("differences", flush=True)
    rgnn.typed_linear(r, dptr, w, dx, trans_w=True)
    rgnn.typed_linear_wgrad(x, r, dptr, dw, workspace(torch.float32, 41, 4, K, N))
    def loss(a, b):
        return float((linear_ref(a, ptr, b, None, 41)[0] * r.double()).sum())
    for i, k in ((0, 0), (8, 23), (9, 5), (40, 11)):
        d = torch.zeros_like(x, dtype=torch.float64)
        d[i, k] = 0.5
        num = loss(x.double() + d, w.double()) - loss(x.double() - d, w.double())
        assert abs(num - float(dx[i, k])) <= 1e-5 * (1 + abs(num))
    for t, k, n in ((0, 0, 0), (1, 3, 3), (2, 23, 19), (3, 4, 7)):
        d = torch.zeros_like(w, dtype=torch.float64)
        d[t, k, n] = 0.5
        num = loss(x.double(), w.double() + d) - loss(x.double(), w.double() - d)
        assert abs(num - float(dw[t, k, n])) <= 1e-5 * (1 + abs(num))


def test_rows_beyond_32_bits():
    """Rows whose byte and element offsets pass 2^32, forward and weight gradient."""
    import torch
    from paper_2301_06284_amd import rgnn
    K, N, rows = 128, 64, (1 << 25) + 4099          # 4.3e9 elements
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    x[-300:] = torch.randn(300, K, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(2, K, N, generator=g, device="cuda").to(torch.bfloat16)
    gather = torch.randint(rows - 300, rows, (500,), generator=g, device="cuda", dtype=torch.int32)
    ptr = [0, 123, 500]
    dptr = torch.tensor(ptr, device="cuda")
    y = torch.zeros(500, N, dtype=torch.bfloat16, device="cuda")
    print("beyond 32 bits", flush=True)
    rgnn.typed_linear(x, dptr, w, y, gather=gather)
    tail, tg = x[-300:], gather - (rows - 300)
    ref, size = linear_ref(tail, ptr, w, tg, 500)
    close(y, ref, size, K)
    dw = torch.zeros(2, K, N, dtype=torch.bfloat16, device="cuda")
    rgnn.typed_linear_wgrad(x, y, dptr, dw, workspace(torch.bfloat16, 500, 2, K, N), gather=gather)
    ref, size = wgrad_ref(tail, y, ptr, tg, None, 2)
    close(dw, ref, size, 377)
    q, s = rgnn.fp8_quantize_rows(x)
    q2, s2 = rgnn.fp8_quantize_rows(tail.contiguous())
    assert torch.equal(q[-300:].view(torch.uint8), q2.view(torch.uint8)) and torch.equal(s[-300:], s2)


# ------------------------------------------------------------------ 8 bits

def power(e):
    """2^e in 64 bits, exactly (torch.ldexp multiplies by a rounded power on the GPU)."""
    import torch
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def fp8_ref(blocks):
    """Blocks [..., n] in 64 bits -> (code values, scale bytes): the least power of two s >= 2^-126
    with max |x| <= 448 s, and x / s rounded to three bits behind the leading one, ties to even."""
    import torch
    top = blocks.abs().amax(dim=-1)
    bad = ~torch.isfinite(top)
    top = torch.where(bad, torch.ones_like(top), top)
    f, e = torch.frexp(top / 448.0)
    e = torch.where(f == 0.5, e - 1, e).clamp(min=-126)
    e = torch.where(top > 0, e, torch.full_like(e, -126))
    x = torch.where(bad[..., None], torch.zeros_like(blocks), blocks) * power(-e[..., None])
    ex = torch.frexp(x)[1].clamp(min=-5)
    step = power(ex - 4)
    q = torch.round(x / step) * step
    return (torch.where(bad[..., None], torch.full_like(q, float("nan")), q),
            torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8))


def same_codes(codes, ref):
    import torch
    got = codes.double()
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got[~nan], ref[~nan])


@pytest.mark.parametrize("K", [1, 16, 100, 128, 129, 500, 512, 640, 1000, 2056])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_fp8_rows(dtype, K):
    """Codes and scales exactly, with rows of zeros, of subnormal and huge values, ties, an
    infinity and a NaN."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt = types()[dtype]
    g = torch.Generator(device="cuda").manual_seed(K)
    x = (torch.randn(37, K, generator=g, device="cuda") * torch.exp(3 * torch.randn(37, 1, generator=g, device="cuda"))).to(dt)
    x[1] = 0
    x[2] = x[2].double().mul(1e-40 if dtype != "fp16" else 1e-7).to(dt)
    x[3] = x[3].sign() * torch.finfo(dt).max
    x[4, 0] = float("inf")
    x[5, -1] = float("nan")
    x[6] = (torch.arange(K, device="cuda") % 60 * 8 + 4).to(dt)   # 448 and ties among them
    wide = torch.full((37, K + 8), float("nan"), dtype=dt, device="cuda")
    wide[:, :K] = x
    print(f"fp8 rows {dtype} {K}", flush=True)
    for src in (x, wide[:, :K]):
        q, s = rgnn.fp8_quantize_rows(src)
        Kp, Ks = rgnn.fp8_widths(K)
        pad = torch.nn.functional.pad(x.double(), (0, Kp - K)).view(37, -1, 128)
        rq, rs = fp8_ref(pad)
        same_codes(q, rq.view(37, Kp))
        assert torch.equal(s[:, :Kp // 128], rs) and (s[:, Kp // 128:] == 127).all()


@pytest.mark.parametrize("K,N", [(1, 1), (128, 128), (100, 77), (136, 264), (520, 200)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_fp8_weights(dtype, K, N):
    import torch
    from paper_2301_06284_amd import rgnn
    dt, T = types()[dtype], 3
    g = torch.Generator(device="cuda").manual_seed(K + N)
    w = (torch.randn(T, K, N, generator=g, device="cuda") * 0.05).to(dt)
    w[1] = 0
    w[2, K // 2, N // 2] = float("nan")
    print(f"fp8 weights {dtype} {K}x{N}", flush=True)
    q, s = rgnn.fp8_quantize_weights(w)
    Kp, Ks = rgnn.fp8_widths(K)
    nb, kb = -(-N // 128), Kp // 128
    pad = torch.nn.functional.pad(w.double(), (0, nb * 128 - N, 0, Kp - K))
    b = pad.view(T, kb, 128, nb, 128).permute(0, 3, 1, 4, 2).reshape(T, nb, kb, -1)     # [.., n * 128 + k]
    rq, rs = fp8_ref(b)
    rq = rq.view(T, nb, kb, 128, 128).permute(0, 1, 3, 2, 4).reshape(T, nb * 128, Kp)[:, :N]
    same_codes(q, rq)
    assert torch.equal(s[:, :, :kb], rs) and (s[:, :, kb:] == 127).all()


def fp8_values(q, s, rows_per_scale):
    import torch
    n, kp = q.shape[-2:]
    e = power(s.int() - 127)[..., :kp // 128]
    e = e.repeat_interleave(rows_per_scale, dim=-2)[..., :n, :].repeat_interleave(128, dim=-1)
    return q.double() * e


@pytest.mark.parametrize("K,N,shape", [(128, 128, "ragged"), (16, 8, "few"), (100, 77, "ragged"), (1000, 264, "few"),
                                       (2048, 520, "dense"), (640, 1100, "one"), (4096, 64, "few")])
@pytest.mark.parametrize("out", ["fp32", "bf16", "fp16"])
def test_fp8_linear(K, N, shape, out):
    import torch
    from paper_2301_06284_amd import rgnn
    ptr = PTRS[shape]
    g, x, w, dptr = case(torch.bfloat16, ptr, K, N, K + N, extra=7)
    M = x.shape[0]
    w[0, : max(1, K // 2)] *= 300                        # blocks of very different scale
    xq, xs = rgnn.fp8_quantize_rows(x)
    wq, ws = rgnn.fp8_quantize_weights(w)
    print(f"fp8 linear {K}x{N} {shape} {out}", flush=True)
    y = torch.full((M, N), 7.0, dtype=types()[out], device="cuda")
    rgnn.typed_linear_fp8(xq, xs, dptr, wq, ws, y)
    xv, wv = fp8_values(xq, xs, 1), fp8_values(wq, ws, 128).transpose(1, 2)
    ref, size = linear_ref(xv, ptr, wv, None, M)
    own = slice(ptr[0], ptr[-1])
    close(y[own], ref[own], size[own], K, grouped=GROUPED)
    assert (y[ptr[-1]:] == 7.0).all() and (y[:ptr[0]] == 7.0).all()
    # gathered rows, outside ones and a scatter
    gather = torch.randint(0, M, (M,), generator=g, device="cuda", dtype=torch.int32)
    scatter = torch.randperm(M, generator=g, device="cuda").to(torch.int32)
    if M > 6:
        gather[4], gather[5] = -1, M
    y.fill_(7.0)
    rgnn.typed_linear_fp8(xq, xs, dptr, wq, ws, y, gather=gather, scatter=scatter)
    ref, size = linear_ref(xv, ptr, wv, gather, M)
    close(y[scatter[own].long()], ref[own], size[own], K, grouped=GROUPED)


@pytest.mark.parametrize("K,N,M", [(128, 16, 16), (384, 264, 70), (1000, 130, 300), (4096, 512, 20)])
def test_fp8_linear_exact(K, N, M):
    """Codes of -4 .. 4 under scales of 1/2, 1 and 2: every product and sum is a multiple of
    1/4 below 2^18, whose bits all fit, so that the fp32 result is exact."""
    import torch
    from paper_2301_06284_amd import rgnn
    g = torch.Generator(device="cuda").manual_seed(K)
    ptr = [0, M // 3, M]
    Kp, Ks = rgnn.fp8_widths(K)
    codes = lambda *s: torch.randint(-4, 5, s, generator=g, device="cuda").float()  # noqa: E731
    scales = lambda *s: torch.randint(126, 129, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    xq, wq = codes(M, Kp), codes(2, N, Kp)
    xq[:, K:], wq[:, :, K:] = 0, 0
    xq, wq = xq.to(torch.float8_e4m3fn), wq.to(torch.float8_e4m3fn)
    xs, ws = scales(M, Ks), scales(2, -(-N // 128), Ks)
    ref, _ = linear_ref(fp8_values(xq, xs, 1), ptr, fp8_values(wq, ws, 128).transpose(1, 2), None, M)
    y = torch.full((M, N), float("nan"), device="cuda")
    print(f"fp8 exact {K}x{N} M={M}", flush=True)
    # K of the call is that of the codes: the last block's codes behind K are zero
    rgnn.typed_linear_fp8(xq, xs, torch.tensor(ptr, device="cuda"), wq, ws, y)
    assert torch.equal(y.double(), ref)


def test_fp8_nan_blocks():
    """A block with a NaN makes its row's outputs NaN and no others."""
    import torch
    from paper_2301_06284_amd import rgnn
    ptr = [0, 40, 90]
    g, x, w, dptr = case(torch.bfloat16, ptr, 300, 136, 4)
    x[7, 130], x[60, 0] = float("inf"), float("nan")
    xq, xs = rgnn.fp8_quantize_rows(x)
    wq, ws = rgnn.fp8_quantize_weights(w)
    y = torch.zeros(90, 136, dtype=torch.bfloat16, device="cuda")
    print("fp8 nan", flush=True)
    rgnn.typed_linear_fp8(xq, xs, dptr, wq, ws, y)
    bad = torch.isnan(y)
    assert bad[7].all() and bad[60].all() and int(bad.sum()) == 2 * 136


# ------------------------------------------------------------------ AdamW

HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


def decode(cm, cv, tm, tv):
    """8-bit states in 64 bits."""
    import torch
    n = cm.numel()
    tm, tv = (t.double().repeat_interleave(256)[:n] for t in (tm, tv))
    a, b = cm.double() / 127, cv.double() / 255
    return a * a.abs() * tm, b ** 4 * tv


def adamw_ref(p, g, m, v, t, scale=1.0, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1):
    p, g, m, v = (x.double() for x in (p, g, m, v))
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p - lr * weight_decay * p - lr * (m / (1 - beta1 ** t)) / ((v / (1 - beta2 ** t)).sqrt() + eps)
    return p, m, v


def near(got, ref, size, what):
    """fp32 results of about ten rounded operations on values up to `size`, then the type's own rounding."""
    t = name_of(got.dtype)
    tol = 16 * 2.0 ** -24 * size + HALF[t] * ref.abs() * 1.001 + LEAST[t]
    worst = float(((got.double() - ref).abs() / tol).max()) if got.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the tolerance"


def check_codes(cm, cv, tm, tv, m, v, size, what):
    """Codes and tops of the 64-bit states m, v; size = beta1 |m before| + (1 - beta1) |g|.
    With u = 2^-24: reading a code c of v rounds 1/255, c/255, its square, that one's square and
    the product with the top, 2 (2 (2 u) + u) + u + u = 12 u; beta2 and the product with it make
    14 u, the sum 15 u (both summands are positive, the other one is nearer).  A first
    moment's code takes 2 (2 u) + u + u = 6 u, beta1 and its product 8 u, the sum 9 u, of `size`,
    since the summands may cancel.  Codes: half a step, for the roundings of quotient, roots and product
    1.1e-4 of one (255 times 15 u / 4 and three more u: 1.03e-4), and what `size` moves them."""
    import torch
    n = m.numel()
    u = 2.0 ** -24
    block = lambda x: torch.nn.functional.pad(x, (0, (-n) % 256)).view(-1, 256)  # noqa: E731
    mb, vb, off = block(m), block(v), 10 * u * block(size)
    rm, rv = mb.abs().amax(1), vb.amax(1)
    assert float(((tm.double() - rm).abs() - off.amax(1)).max()) <= 2.0 ** -149, what
    assert float(((tv.double() - rv).abs() - 16 * u * rv).max()) <= 2.0 ** -149, what
    cm, cv = block(cm).double(), block(cv).double()
    code = lambda x: 127 * (x.clamp(min=0) / rm.clamp(min=1e-300)[:, None]).sqrt()  # noqa: E731
    c, sure = cm * torch.sign(mb), mb.abs() > off          # the sign of a cancelled moment is open
    c = torch.where(sure, c, cm.abs())
    low, high = code(mb.abs() - 2 * off), code(mb.abs() + 2 * off)
    assert float(torch.maximum(low - c, c - high).max()) <= 0.5 + 1.1e-4, what
    iv = 255 * (vb / rv.clamp(min=1e-300)[:, None]) ** 0.25
    dv = (cv - iv).abs()
    assert float(torch.where((cv == 1) & (iv < 1), torch.zeros_like(dv), dv).max()) <= 0.5 + 1.1e-4, what
    assert not ((cv == 0) & (vb > 0)).any(), f"{what}: a second moment became zero"
    assert not ((cv != 0) & (vb == 0)).any(), what


def states(sizes, ptype, gtype, bits, copy, seed, offset=0):
    """Lists of tensors, each `offset` elements behind an aligned address."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    def make(n, dt, f):
        buf = torch.zeros(n + offset + 4, dtype=dt, device="cuda")
        out = buf[offset:offset + n]
        out.copy_(f(torch.randn(n, generator=gen, device="cuda")).to(dt))
        return out
    d = dict(params=[], grads=[], m=[], v=[])
    if bits == 8:
        d.update(m_scale=[], v_scale=[])
    if copy:
        d.update(copies=[])
    for n in sizes:
        d["params"].append(make(n, ptype, lambda x: x * 0.05))
        d["grads"].append(make(n, gtype, lambda x: x * 0.01))
        if bits == 8:
            blocks = -(-n // 256)
            d["m"].append(make(n, torch.int8, lambda x: (x * 40).clamp(-127, 127).round()))
            d["v"].append(make(n, torch.uint8, lambda x: (128 + x * 40).clamp(0, 255).round()))
            d["m_scale"].append(make(blocks, torch.float32, lambda x: torch.exp(x) * 1e-3))
            d["v_scale"].append(make(blocks, torch.float32, lambda x: torch.exp(x) * 1e-4))
        else:
            d["m"].append(make(n, torch.float32, lambda x: x * 1e-3))
            d["v"].append(make(n, torch.float32, lambda x: x * x * 1e-5))
        if copy:
            d["copies"].append(make(n, copy, lambda x: x * 0))
    return d


SIZES = [1, 3, 255, 256, 257, 4095, 4096, 4097, 30001, 0, 77]


def check_step(d, old, t, bits, scale=1.0, hyper=None):
    """Every tensor of `d` after one step against the 64-bit step of `old`."""
    hyper = hyper or HYPER
    for i in range(len(d["params"])):
        if d["params"][i].numel() == 0:
            continue
        om, ov = (decode(*(old[k][i] for k in ("m", "v", "m_scale", "v_scale"))) if bits == 8 else
                  (old["m"][i], old["v"][i]))
        p, m, v = adamw_ref(old["params"][i], old["grads"][i], om, ov, t, scale, **hyper)
        step = hyper["lr"] * (m / (1 - hyper["beta1"] ** t)).abs() / ((v / (1 - hyper["beta2"] ** t)).sqrt() + hyper["eps"])
        near(d["params"][i], p, old["params"][i].double().abs() + step, f"param {i}")
        if "copies" in d:
            near(d["copies"][i], p, old["params"][i].double().abs() + step, f"copy {i}")
        if bits == 8:
            size = hyper["beta1"] * om.abs() + (1 - hyper["beta1"]) * old["grads"][i].double().abs() * scale
            check_codes(d["m"][i], d["v"][i], d["m_scale"][i], d["v_scale"][i], m, v, size, f"tensor {i}")
        else:
            g = old["grads"][i].double().abs() * scale
            near(d["m"][i], m, om.double().abs() + g, f"m {i}")
            near(d["v"][i], v, v, f"v {i}")


def clone(d):
    return {k: [x.clone() for x in v] for k, v in d.items()}


@pytest.mark.parametrize("ptype,gtype,copy", [("fp32", "fp32", None), ("fp32", "bf16", "bf16"), ("fp32", "fp16", "fp16"),
                                              ("bf16", "bf16", None), ("bf16", "fp32", "fp32"), ("fp16", "fp16", None),
                                              ("fp16", "bf16", None), ("bf16", "fp16", None), ("fp16", "fp32", None)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
def test_adamw(ptype, gtype, copy, bits, offset):
    import torch
    from paper_2301_06284_amd import rgnn
    ts = types()
    d = states(SIZES, ts[ptype], ts[gtype], bits, ts[copy] if copy else None, 11, offset)
    old = clone(d)
    print(f"adamw {ptype} {gtype} {copy} bits={bits} offset={offset}", flush=True)
    rgnn.adamw_step(rgnn.AdamwTensors(**d), 7, **HYPER)
    torch.cuda.synchronize()
    check_step(d, old, 7, bits)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_many_tensors_of_mixed_types(bits):
    """More tensors than one launch takes, of several type combinations in turn, in neither
    address nor size order; a gradient factor and a step number that lie on the device."""
    import torch
    from paper_2301_06284_amd import rgnn
    ts = types()
    rng = np.random.default_rng(bits)
    sizes = [int(s) for s in np.exp(rng.uniform(0, 9, 200))]
    parts = [states(sizes[k::3], ts[p], ts[g], bits, None, k) for k, (p, g) in
             enumerate((("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")))]
    d = {k: [t for part in parts for t in part[k]] for k in parts[0]}
    order = rng.permutation(len(d["params"]))
    d = {k: [v[i] for i in order] for k, v in d.items()}
    old = clone(d)
    step = torch.tensor([3], device="cuda")
    factor = torch.tensor([0.25], device="cuda")
    print(f"adamw many bits={bits}", flush=True)
    rgnn.adamw_step(rgnn.AdamwTensors(**d), step, grad_scale=factor, **HYPER)
    torch.cuda.synchronize()
    check_step(d, old, 3, bits, 0.25)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_from_zero_states(bits):
    """The first step from zero states, zero gradients among them, then a second: nothing is
    divided by zero, and a parameter without gradient only decays."""
    import torch
    from paper_2301_06284_amd import rgnn
    ts = types()
    d = states([1000], ts["fp32"], ts["fp32"], bits, None, 3)
    for k in ("m", "v", "m_scale", "v_scale"):
        for x in d.get(k, []):
            x.zero_()
    d["grads"][0][300:700] = 0
    tensors = rgnn.AdamwTensors(**d)
    print(f"adamw zero bits={bits}", flush=True)
    for t in (1, 2):
        old = clone(d)
        rgnn.adamw_step(tensors, t, **HYPER)
        torch.cuda.synchronize()
        check_step(d, old, t, bits)
        assert torch.isfinite(d["params"][0]).all()


@pytest.mark.parametrize("hyper", [dict(lr=0.5, beta1=0.0, beta2=0.0, eps=1e-3, weight_decay=0.0),
                                   dict(lr=0.0, beta1=0.9, beta2=0.95, eps=0.1, weight_decay=0.3),
                                   dict(lr=-1e-3, beta1=0.5, beta2=0.5, eps=1e-6, weight_decay=0.1)])
@pytest.mark.parametrize("on_device", [False, True])
def test_adamw_hyper_parameters(hyper, on_device):
    import torch
    from paper_2301_06284_amd import rgnn
    d = states([513], torch.float32, torch.float32, 32, None, 8)
    old = clone(d)
    hyper = dict(hyper)
    print(f"adamw hyper {hyper} {on_device}", flush=True)
    rgnn.adamw_step(rgnn.AdamwTensors(**d), torch.tensor([10 ** 9], device="cuda") if on_device else 10 ** 9, **hyper)
    torch.cuda.synchronize()
    p, m, v = adamw_ref(old["params"][0], old["grads"][0], old["m"][0], old["v"][0], 10 ** 9, **hyper)
    size = old["params"][0].double().abs() + abs(hyper["lr"]) * m.abs() / (v.sqrt() + hyper["eps"])
    near(d["params"][0], p, size, "param")


def test_adamw_empty_list():
    from paper_2301_06284_amd import rgnn
    rgnn.adamw_step(rgnn.AdamwTensors([], [], [], []), 1, 1e-3)


# ------------------------------------------------------------------ together

def train_step(x, dptr, w16, master, y, target, dy, dx, dw, work, tensors, step):
    """One training step of the typed linear on a squared error, with the library's calls
    and one elementwise operation."""
    import torch
    from paper_2301_06284_amd import rgnn
    rgnn.typed_linear(x, dptr, w16, y)
    torch.sub(y, target, out=dy)
    rgnn.typed_linear(dy, dptr, w16, dx, trans_w=True)
    rgnn.typed_linear_wgrad(x, dy, dptr, dw, work)
    rgnn.adamw_step(tensors, step, **HYPER)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("K,N", [(64, 64), (264, 136)])
def test_train_and_serve(bits, K, N):
    """Three training steps in 16 bits with fp32 parameters, eager, on another stream and
    as a captured graph replayed between eager work; the three agree bit for bit.  Then the
    trained weights in 8 bits against the product of their codes in 64."""
    import torch
    from paper_2301_06284_amd import rgnn
    ptr = [0, 50, 50, 333, 700]
    dt, T, M = torch.bfloat16, 4, 720
    results = []
    for mode in ("eager", "stream", "graph"):
        g, x, w, dptr = case(dt, ptr, K, N, 21, extra=20)
        target = torch.randn(M, N, generator=g, device="cuda").to(dt)
        master = w.float()
        w16 = w.clone()
        y, dy = torch.zeros(M, N, dtype=dt, device="cuda"), torch.zeros(M, N, dtype=dt, device="cuda")
        dx, dw = torch.zeros(M, K, dtype=dt, device="cuda"), torch.zeros(T, K, N, dtype=dt, device="cuda")
        n = w.numel()
        st = dict(m=[torch.zeros(n, dtype=torch.float32 if bits == 32 else torch.int8, device="cuda")],
                  v=[torch.zeros(n, dtype=torch.float32 if bits == 32 else torch.uint8, device="cuda")])
        if bits == 8:
            st.update(m_scale=[torch.zeros(-(-n // 256), device="cuda")], v_scale=[torch.zeros(-(-n // 256), device="cuda")])
        tensors = rgnn.AdamwTensors([master.view(-1)], [dw.view(-1)], copies=[w16.view(-1)], **st)
        work = workspace(dt, M, T, K, N)
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        args = (x, dptr, w16, master, y, target, dy, dx, dw, work, tensors, step)
        print(f"train {mode} bits={bits} {K}x{N}", flush=True)
        if mode == "eager":
            for _ in range(3):
                step += 1
                train_step(*args)
        elif mode == "stream":
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                for _ in range(3):
                    step += 1
                    train_step(*args)
            torch.cuda.current_stream().wait_stream(s)
        else:
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step += 1
                train_step(*args)
            assert int(step) == 0                       # captured, not run
            other = torch.zeros(M, N, dtype=dt, device="cuda")
            for _ in range(3):
                graph.replay()
                rgnn.typed_linear(x, dptr, w, other)    # eager work between the replays
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        results.append([t.clone() for t in (master, w16, y, dx, dw, st["m"][0], st["v"][0])])
    for a, b, c in zip(*results):
        assert torch.equal(a, b) and torch.equal(a, c)
    master, w16 = results[0][0], results[0][1]
    assert not torch.equal(w16, w) and torch.equal(master.to(dt), w16)
    wq, ws = rgnn.fp8_quantize_weights(w16)
    xq, xs = rgnn.fp8_quantize_rows(x)
    y8 = torch.zeros(M, N, dtype=dt, device="cuda")
    rgnn.typed_linear_fp8(xq, xs, dptr, wq, ws, y8)
    ref, size = linear_ref(fp8_values(xq, xs, 1), ptr, fp8_values(wq, ws, 128).transpose(1, 2), None, M)
    close(y8[:700], ref[:700], size[:700], K, grouped=GROUPED)


def test_segment_gemm_agrees():
    """fp32 at the segment GEMM's widths: the typed linear over the same offsets on the
    device gives its results within fp32's accuracy."""
    import torch
    from paper_2301_06284_amd import rgnn
    ptr, K, N = PTRS["ragged"], 64, 128
    g, x, w, dptr = case(torch.float32, ptr, K, N, 6)
    a, b = torch.zeros(1000, N, device="cuda"), torch.zeros(1000, N, device="cuda")
    ws = torch.empty(rgnn.segment_gemm_workspace_size(1000, 6), dtype=torch.uint8, device="cuda")
    rgnn.segment_gemm(x, None, np.array(ptr), w, a, None, ws, K, N)
    rgnn.typed_linear(x, dptr, w, b)
    ref, size = linear_ref(x, ptr, w, None, 1000)
    close(a, ref, size, K)
    close(b, ref, size, K)


def test_two_streams_at_once():
    """Two weight gradients at once on two streams with a workspace each."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, ptr, K, N = torch.bfloat16, [0, 20000, 26000], 64, 64
    g, x, w, dptr = case(dt, ptr, K, N, 31)
    dy = [torch.randn(26000, N, generator=g, device="cuda").to(dt) for _ in range(2)]
    alone = []
    for d in dy:
        dw = torch.zeros(2, K, N, dtype=dt, device="cuda")
        rgnn.typed_linear_wgrad(x, d, dptr, dw, workspace(dt, 26000, 2, K, N))
        alone.append(dw)
    both = [torch.zeros(2, K, N, dtype=dt, device="cuda") for _ in range(2)]
    works = [workspace(dt, 26000, 2, K, N) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    print("two streams", flush=True)
    for _ in range(3):
        for k in range(2):
            rgnn.typed_linear_wgrad(x, dy[k], dptr, both[k], works[k], stream=streams[k])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, both))


@pytest.mark.parametrize("ptr", [[0, 700, 300, 900, 900, 1000], [500, -7, 1200, 3, 800, 5000], [0] * 3 + [900] + [100] * 300 + [1000],
                                 [40] + [0, 2 ** 62] * 300])
def test_offsets_that_descend(ptr):
    """Offsets are kept inside [0, M], and one below an earlier one counts as that: forward, weight
    gradient and 8 bits as with the running maximum."""
    import torch
    from paper_2301_06284_amd import rgnn
    M, K, N, T = 1000, 136, 72, len(ptr) - 1
    kept = np.maximum.accumulate(np.clip(np.array(ptr), 0, M)).tolist()
    g, x, w, dkept = case(torch.bfloat16, kept, K, N, T, extra=M - kept[-1])
    given = torch.tensor(ptr, dtype=torch.int64, device="cuda")
    xq, xs = rgnn.fp8_quantize_rows(x)
    wq, ws = rgnn.fp8_quantize_weights(w)
    print(f"descending offsets {T}", flush=True)
    out = []
    for p in (given, dkept):
        y, y8 = (torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        dw = torch.full((T, K, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        rgnn.typed_linear(x, p, w, y)
        rgnn.typed_linear_fp8(xq, xs, p, wq, ws, y8)
        rgnn.typed_linear_wgrad(x, x[:, :N], p, dw, workspace(torch.bfloat16, M, T, K, N))
        out.append((y, y8, dw))
    ref, size = linear_ref(x, kept, w, None, M)
    close(out[1][0][kept[0]:kept[-1]], ref[kept[0]:kept[-1]], size[kept[0]:kept[-1]], K)
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("K,N", [(64, 64), (91, 80), (264, 136)])
def test_wgrad_of_rows_outside(dtype, K, N):
    """A position whose row of X or of dY lies outside adds nothing, whatever the other row holds."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, ptr, rows = types()[dtype], [0, 90, 90, 700, 3000], 500
    M, T = ptr[-1], 4
    g = torch.Generator(device="cuda").manual_seed(K)
    x, dy = (torch.randn(rows, c, generator=g, device="cuda").to(dt) for c in (K, N))
    x[3], dy[5] = float("nan"), float("inf")
    gather, dyg = (torch.randint(6, rows, (M,), generator=g, device="cuda", dtype=torch.int32) for _ in range(2))
    for k, (a, b) in enumerate([(-1, 5), (3, rows), (rows + 9, 5), (3, -8)]):
        gather[k::97], dyg[k::97] = a, b
    print(f"wgrad of rows outside {dtype} {K}x{N}", flush=True)
    dw = torch.full((T, K, N), float("nan"), dtype=dt, device="cuda")
    rgnn.typed_linear_wgrad(x, dy, torch.tensor(ptr, device="cuda"), dw, workspace(dt, M, T, K, N), gather=gather, dy_gather=dyg)
    inside = (gather > 5) & (gather < rows) & (dyg > 5) & (dyg < rows)
    sel = torch.where(inside, gather, torch.full_like(gather, -1))
    x[3], dy[5] = 0.0, 0.0
    ref, size = wgrad_ref(x, dy, ptr, sel, dyg, T)
    close(dw, ref, size, 2300)


def test_typed_linear_of_no_rows():
    """X without rows, reached through an index array: zeros; and a gradient of no positions: zeros."""
    import torch
    from paper_2301_06284_amd import rgnn
    dt, K, N = torch.bfloat16, 256, 128
    w = torch.randn(2, K, N, device="cuda").to(dt)
    none = torch.empty(0, K, dtype=dt, device="cuda")
    ptr = torch.tensor([0, 3, 40], device="cuda")
    gather = torch.zeros(40, dtype=torch.int32, device="cuda")
    y = torch.full((40, N), float("nan"), dtype=dt, device="cuda")
    print("no rows", flush=True)
    rgnn.typed_linear(none, ptr, w, y, gather=gather)
    assert (y == 0).all()
    dw = torch.full((2, K, N), float("nan"), dtype=dt, device="cuda")
    rgnn.typed_linear_wgrad(none, torch.empty(0, N, dtype=dt, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), dw, None)
    assert (dw == 0).all()


def test_wide_tile_near_32_bits():
    """Rows whose byte offsets lie just below 2^32, where the widest tile takes 32-bit offsets from the matrix, and
    beyond, where it does not: the same bits as the same rows of a small matrix."""
    import torch
    from paper_2301_06284_amd import rgnn
    K, N, M = 2048, 4096, 16384
    g = torch.Generator(device="cuda").manual_seed(9)
    tail = torch.randn(1000, K, generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn(1, K, N, generator=g, device="cuda") / 45).to(torch.bfloat16)
    index = torch.randint(0, 1000, (M,), generator=g, device="cuda", dtype=torch.int32)
    ptr = torch.tensor([0, M], device="cuda")
    ref = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    rgnn.typed_linear(tail, ptr, w, ref, gather=index)
    for rows in ((1 << 20) - 1, (1 << 20) + 700):      # 4096 bytes each
        x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
        x[-1000:] = tail
        y = torch.full((M, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        print(f"wide tile, {rows} rows", flush=True)
        rgnn.typed_linear(x, ptr, w, y, gather=index + (rows - 1000))
        size = (tail.double().abs().mean() * 0.02 * K).item()
        assert (y.double() - ref.double()).abs().max().item() <= 2 * (K * 2.0 ** -23 * size + 2.0 ** -8 * ref.double().abs().max().item())
        if rows < 1 << 20:
            assert torch.equal(y, ref)
        # positions far into the matrix, without an index array for X
        at = rows - 1000
        far = torch.tensor([at, rows], device="cuda")
        scatter = torch.arange(-at, rows - at, dtype=torch.int32, device="cuda")
        z = torch.full((1000, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        rgnn.typed_linear(x, far, w, z, scatter=scatter)
        first = torch.full((1000, N), float("nan"), dtype=torch.bfloat16, device="cuda")
        rgnn.typed_linear(tail, torch.tensor([0, 1000], device="cuda"), w, first)
        assert (z.double() - first.double()).abs().max().item() <= 2 * (K * 2.0 ** -23 * size + 2.0 ** -8 * first.double().abs().max().item())
        del x, y, z


def test_more_workgroups_than_a_launch_is_wide():
    """2^24 workgroups and more: rows of one column, and rows in 8 bits."""
    import torch
    from paper_2301_06284_amd import rgnn
    rows = (1 << 30) + 777
    x = torch.empty(rows, 1, device="cuda")
    part = torch.arange(1 << 20, device="cuda", dtype=torch.float32)
    x[:1 << 30].view(1 << 10, 1 << 20).copy_(part)
    x[1 << 30:, 0] = part[:777] + 5
    cut = (1 << 30) + 100
    y = torch.empty(rows, 1, device="cuda")
    print("2^30 rows", flush=True)
    rgnn.typed_linear(x, torch.tensor([0, cut, rows], device="cuda"), torch.tensor([2.0, -4.0], device="cuda").view(2, 1, 1), y)
    x[:cut] *= 2
    x[cut:] *= -4
    assert torch.equal(x, y)
    del x, y
    rows = (1 << 26) + 9
    x = torch.empty(rows, 8, dtype=torch.bfloat16, device="cuda")
    x[:] = torch.tensor([1.0, -2, 3, 0.5, 0, 7, -448, 5], device="cuda").to(torch.bfloat16)
    x[-9:] *= 2
    print("2^26 rows in 8 bits", flush=True)
    codes, scales = rgnn.fp8_quantize_rows(x)
    first = codes[:1].view(torch.uint8)
    assert (scales[:-9, 0] == 127).all() and (scales[-9:, 0] == 128).all() and (scales[:, 1:] == 127).all()
    for at in range(0, rows, 1 << 24):
        assert (codes[at:at + (1 << 24)].view(torch.uint8) == first).all()


def test_quantize_on_another_stream():
    """Outputs made by the call belong to the stream that writes them: memory that the current stream has
    given back with work still under way is not theirs."""
    import torch
    from paper_2301_06284_amd import rgnn
    x = torch.randn(4096, 512, device="cuda").to(torch.bfloat16)
    ref = rgnn.fp8_quantize_rows(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    print("quantize on another stream", flush=True)
    for stream in (side, side.cuda_stream, 0):
        for _ in range(3):
            busy = torch.empty(4096, 512, dtype=torch.uint8, device="cuda")   # the codes' size
            for _ in range(20):
                busy.fill_(3)                                                 # under way on the current stream
            del busy
            codes, scales = rgnn.fp8_quantize_rows(x, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(codes.view(torch.uint8), ref[0].view(torch.uint8)) and torch.equal(scales, ref[1])
