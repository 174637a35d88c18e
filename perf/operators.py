"""Performance cases of the typed linear's training and serving operators: the
typed linear over ragged segments whose offsets lie on the device (forward,
input gradient, weight gradient; fp32, bf16, fp16), its 8-bit form with a scale
for each block of 128, and the AdamW step over many tensors with states in 32
or in 8 bits.

A case names an operation (`op`):

  linear    Y[scatter[i]] = X[gather[i]] W[t(i)], rows of one type contiguous
  step      the same with its two gradients: dX = dY W^T and dW[t] = X_t^T dY_t
  fp8       rows quantised to 8 bits, then the product with weights kept in 8 bits
  fp8_new   the same with the weights quantised in the pass too (new weights)
  adamw     one AdamW step of all tensors of a model

`run` computes them in elementary torch operations in 32 bits, or (where `own`)
with the calls of paper_2301_06284_amd.rgnn.

Types' sizes follow a Zipf law of exponent `skew` over a fixed shuffle; they
depend on the case alone, the values on the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
BLOCK = 128       # elements of one 8-bit scale along K (and along N for weights)
QBLOCK = 256      # elements of one block of 8-bit optimizer states
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def listed():
    return [
        # serving, single tokens: 8 tokens, two of 32 weights each; the weights' bytes
        dict(name="linear_tokens", op="linear", dtype="bf16", M=16, X=8, T=32, K=2048, N=1536, skew=0.0, index=True),
        # a graph layer's messages: gathered and scattered rows, narrow weights
        dict(name="linear_relations", op="linear", dtype="bf16", M=1000003, X=600011, T=96, K=64, N=128, skew=1.2,
             index=True),
        # a long prompt through wide weights: the matrix cores
        dict(name="linear_prompt", op="linear", dtype="bf16", M=16384, X=8192, T=32, K=2048, N=4096, skew=0.4,
             index=True),
        # a training step of wide weights
        dict(name="step_wide", op="step", dtype="bf16", M=8192, X=8192, T=16, K=2048, N=1536, skew=0.4, index=False),
        # a training step of a graph layer in fp16
        dict(name="step_relations", op="step", dtype="fp16", M=300007, X=300007, T=96, K=64, N=64, skew=1.2,
             index=False),
        # fp32 with feature widths that fill no vector and no tile
        dict(name="step_odd_f32", op="step", dtype="fp32", M=10007, X=10007, T=7, K=100, N=77, skew=0.8, index=False),
        # serving in 8 bits: single tokens
        dict(name="fp8_tokens", op="fp8", dtype="bf16", M=16, X=8, T=32, K=2048, N=1536, skew=0.0, index=True),
        # one dense weight, a long prompt
        dict(name="fp8_dense", op="fp8", dtype="bf16", M=8192, X=8192, T=1, K=4096, N=4096, skew=0.0, index=False),
        # after an update of the weights: they are quantised again, then used
        dict(name="fp8_new_weights", op="fp8_new", dtype="bf16", M=4099, X=4099, T=16, K=2048, N=1536, skew=0.4,
             index=False),
        # the seven tensors of an HGT layer (4 node types, 7 relations, d = 64, 4 heads): latency
        dict(name="adamw_hgt", op="adamw", dtype="fp32", grad="fp32", bits=32, copy="", shape="hgt", n=77831),
        # a few hundred tensors from one value to a million, 16-bit parameters
        dict(name="adamw_many", op="adamw", dtype="bf16", grad="bf16", bits=32, copy="", shape="many", n=24000000),
        # wide weights of many types: states in 8 bits, 16-bit gradients and working copy
        dict(name="adamw_8bit", op="adamw", dtype="fp32", grad="bf16", bits=8, copy="bf16", shape="wide", n=201326592),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A feature width: mostly whole vectors of 16 bytes, one in four any number."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)


def draw(rng):
    op = rng.choice(["linear", "linear", "step", "step", "fp8", "fp8_new", "adamw", "adamw"])
    if op == "adamw":
        shape = rng.choice(["hgt", "many", "wide"])
        n = _log_int(rng, 1000, {"hgt": 1000000, "many": 30000000, "wide": 100000000}[shape])
        dtype = rng.choice(["fp32", "fp32", "bf16", "fp16"])
        return dict(op=op, dtype=dtype, grad=rng.choice(["fp32", "bf16"]) if dtype == "fp32" else dtype,
                    bits=rng.choice([32, 8]), copy=rng.choice(["", "bf16"]) if dtype == "fp32" else "", shape=shape, n=n)
    t = _log_int(rng, 1, 128)
    if rng.random() < 0.4:    # graph layers: many rows, narrow weights
        m, k, n = _log_int(rng, 1000, 600000), _width(rng, 16, 160), _width(rng, 16, 160)
        skew = rng.uniform(0.0, 1.3)
    else:                     # experts: few rows or many, wide weights
        m, k, n = _log_int(rng, 1, 8192), _width(rng, 128, 3000), _width(rng, 128, 3000)
        t, skew = min(t, 64), rng.uniform(0.0, 0.6)
        if op != "linear":
            t = min(t, 32)
    index = rng.random() < 0.5 if op != "step" else False
    x = max(1, int(m * rng.uniform(0.4, 1.2))) if index else m
    return dict(op=op, dtype="bf16" if op.startswith("fp8") else rng.choice(["bf16", "bf16", "fp16", "fp32"]), M=m, X=x,
                T=t, K=k, N=n, skew=round(skew, 2), index=index)


# ------------------------------------------------------------------ inputs

def _sizes(case):
    """Rows of each type: a multinomial draw of Zipf shares, the same for every seed."""
    r = np.random.RandomState(7 + case["M"] + 13 * case["T"])
    p = 1.0 / np.arange(1, case["T"] + 1) ** case["skew"]
    r.shuffle(p)
    return r.multinomial(case["M"], p / p.sum())


def _tensor_sizes(case):
    """Elements of each parameter tensor of an AdamW case."""
    n = case["n"]
    if case["shape"] == "hgt":       # four weights of 4 types, two of 7 relations, one prior
        a, b = max(1, n * 16384 // 77831), max(1, n * 1792 // 77831)
        return [a, a, a, a, b, b, max(1, n - 4 * a - 2 * b)]
    if case["shape"] == "wide":      # two stacked weights, a router and two vectors
        return [max(1, n // 2), max(1, n // 2 - n // 64), max(1, n // 64 - 4100), 2048, 1]
    r = random.Random(n)
    share = [math.exp(r.uniform(0.0, math.log(1e6))) for _ in range(230)]
    return [max(1, int(n * s / sum(share))) for s in share]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _kp(k):
    return -(-k // BLOCK) * BLOCK


def _ks(k):
    return -(-k // (4 * BLOCK)) * 4


def prepare(case, seed):
    g = _gen(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    if case["op"] == "adamw":
        return _prepare_adamw(case, randn, seed)
    dt, m, k, n, t = DT[case["dtype"]], case["M"], case["K"], case["N"], case["T"]
    sizes = _sizes(case)
    ptr = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    # rows of very different size, as activations have
    x = (randn(case["X"], k) * torch.exp(randn(case["X"], 1))).to(dt)
    s = dict(case=case, x=x, host_ptr=ptr.tolist(), ptr=torch.from_numpy(ptr).cuda(), gather=None, scatter=None)
    w = randn(t, k, n).mul_(1.0 / math.sqrt(k)).to(dt)
    if case["index"]:
        s["gather"] = torch.randint(0, case["X"], (m,), generator=g, device="cuda", dtype=torch.int32)
        s["scatter"] = torch.randperm(m, generator=g, device="cuda").to(torch.int32)
    if case["op"] == "step":
        s["dy"] = (randn(m, n) * 0.01).to(dt)
    if case["op"] == "fp8":
        s["wq"], s["ws"] = _quantize_weights(w)
    else:
        s["w"] = w
    return s


def _prepare_adamw(case, randn, seed):
    """Every tensor starts at a multiple of 256 elements of one flat buffer per
    kind, as an allocator places them; the gaps are zero and stay so."""
    sizes = _tensor_sizes(case)
    at, total = [], 0
    for n in sizes:
        at.append((total, n))
        total += -(-n // QBLOCK) * QBLOCK
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    for o, n in at:
        used[o:o + n] = True
    scale = torch.exp(randn(total // QBLOCK, 1)).expand(-1, QBLOCK).reshape(-1)
    p = randn(total).mul_(0.02).mul_(used).to(DT[case["dtype"]])
    grad = randn(total).mul_(1e-3).mul_(scale).mul_(used).to(DT[case["grad"]])
    m = randn(total).mul_(3e-4).mul_(scale).mul_(used)
    v = randn(total).square_().add_(0.05).mul_(1e-6).mul_(scale).mul_(scale).mul_(used)
    s = dict(case=case, at=at, p=p, grad=grad, step=1000 + seed % 7)
    if case["bits"] == 8:
        s["m"], s["ms"] = _encode_m(m)
        s["v"], s["vs"] = _encode_v(v)
    else:
        s["m"], s["v"] = m, v
    if case["copy"]:
        s["copy"] = torch.zeros(total, dtype=DT[case["copy"]], device="cuda")
    return s


# ------------------------------------------------------------------ plain forms

def _rows(s):
    """The rows in type order, in 32 bits."""
    x = s["x"].float()
    return x if s["gather"] is None else x[s["gather"].long()]


def _place(s, y, dt):
    """Rows in type order to their places, rounded once."""
    y = y.to(dt)
    if s["scatter"] is None:
        return y
    out = torch.empty_like(y)
    out[s["scatter"].long()] = y
    return out


def _products(ptr, a, w):
    """a[rows of t] @ w[t] for every type that has rows."""
    out = torch.empty(a.shape[0], w.shape[2], dtype=a.dtype, device=a.device)
    for t in range(w.shape[0]):
        if ptr[t + 1] > ptr[t]:
            torch.matmul(a[ptr[t]:ptr[t + 1]], w[t], out=out[ptr[t]:ptr[t + 1]])
    return out


def _outer(ptr, a, b, types):
    """a[rows of t]^T @ b[rows of t]; zero for a type without rows."""
    out = torch.zeros(types, a.shape[1], b.shape[1], dtype=a.dtype, device=a.device)
    for t in range(types):
        if ptr[t + 1] > ptr[t]:
            torch.matmul(a[ptr[t]:ptr[t + 1]].t(), b[ptr[t]:ptr[t + 1]], out=out[t])
    return out


def _scale_bytes(top):
    """The biased exponent of the least power of two s with top <= 448 s (at least 2^-126),
    from the bits of the largest magnitude `top` (fp32)."""
    bits = top.view(torch.int32)
    return (((bits + 0x1FFFFF) >> 23) - 8).clamp(1, 254)


def _quantize_rows(x):
    """[rows, K] -> codes [rows, Kp] and scale bytes [rows, Ks] (127, a scale of 1, behind the last block)."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x.float(), (0, _kp(k) - k)).view(rows, -1, BLOCK)
    e = _scale_bytes(x.abs().amax(dim=2))
    q = (x * torch.exp2((127 - e).float()).unsqueeze(2)).view(rows, -1).to(torch.float8_e4m3fn)
    return q, torch.nn.functional.pad(e, (0, _ks(k) - e.shape[1]), value=127).to(torch.uint8)


def _quantize_weights(w):
    """[T, K, N] -> codes [T, N, Kp] and scale bytes [T, ceil(N / 128), Ks], a scale for each 128 x 128 block."""
    t, k, n = w.shape
    np_ = _kp(n)
    x = torch.nn.functional.pad(w.float(), (0, np_ - n, 0, _kp(k) - k)).transpose(1, 2)
    x = x.reshape(t, np_ // BLOCK, BLOCK, -1, BLOCK)
    e = _scale_bytes(x.abs().amax(dim=(2, 4)))
    q = (x * torch.exp2((127 - e).float())[:, :, None, :, None]).view(t, np_, -1)[:, :n]
    return q.to(torch.float8_e4m3fn).contiguous(), torch.nn.functional.pad(e, (0, _ks(k) - e.shape[2]),
                                                                          value=127).to(torch.uint8)


def _read_rows(q, e):
    """The values that codes and row scales stand for, in 32 bits."""
    rows, kp = q.shape
    s = torch.exp2(e[:, :kp // BLOCK].float() - 127)
    return (q.float().view(rows, -1, BLOCK) * s.unsqueeze(2)).view(rows, kp)


def _read_weights(q, e):
    """[T, Kp, N] in 32 bits."""
    t, n, kp = q.shape
    s = torch.exp2(e[:, :, :kp // BLOCK].float() - 127).repeat_interleave(BLOCK, dim=1)[:, :n]
    return (q.float().view(t, n, -1, BLOCK) * s.unsqueeze(3)).view(t, n, kp).transpose(1, 2).contiguous()


def _encode_m(m):
    """Signed first moments: code = sign * round(127 sqrt(|m| / top)) of blocks of 256, top their largest magnitude."""
    b = m.view(-1, QBLOCK)
    top = b.abs().amax(dim=1, keepdim=True)
    part = torch.where(top > 0, b.abs() / top, torch.zeros_like(b))
    return (torch.round(127.0 * torch.sqrt(part)) * torch.sign(b)).to(torch.int8).view(-1), top.view(-1)


def _encode_v(v):
    """Second moments: code = round(255 (v / top)^(1/4)), at least 1 where v > 0, so that none becomes zero."""
    b = v.view(-1, QBLOCK)
    top = b.amax(dim=1, keepdim=True)
    part = torch.where(top > 0, b / top, torch.zeros_like(b))
    code = torch.round(255.0 * torch.sqrt(torch.sqrt(part)))
    return torch.maximum(code, (b > 0).to(code.dtype)).to(torch.uint8).view(-1), top.view(-1)


def _decode_m(c, top):
    f = c.to(top.dtype).view(-1, QBLOCK) * (1.0 / 127.0)
    return (f * f.abs() * top[:, None]).view(-1)


def _decode_v(c, top):
    f = c.to(top.dtype).view(-1, QBLOCK) * (1.0 / 255.0)
    f = f * f
    return (f * f * top[:, None]).view(-1)


def _adamw_plain(s):
    eight = s["case"]["bits"] == 8
    g, p = s["grad"].float(), s["p"].float()
    m = _decode_m(s["m"], s["ms"]) if eight else s["m"]
    v = _decode_v(s["v"], s["vs"]) if eight else s["v"]
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    denom = torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** s["step"])) + EPS
    p = p * (1 - LR * DECAY) - (m / denom) * (LR / (1 - BETA1 ** s["step"]))
    s["p"].copy_(p)
    if "copy" in s:
        s["copy"].copy_(p)
    if eight:
        (s["m"], s["ms"]), (s["v"], s["vs"]) = _encode_m(m), _encode_v(v)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def _adamw_own(s):
    from paper_2301_06284_amd import rgnn
    if "tensors" not in s:      # a program keeps its tensors' list
        cut = lambda b: [b[o:o + n] for o, n in s["at"]]  # noqa: E731
        cut_top = lambda b: [b[o // QBLOCK:-(-(o + n) // QBLOCK)] for o, n in s["at"]]  # noqa: E731
        views = dict(params=cut(s["p"]), grads=cut(s["grad"]), m=cut(s["m"]), v=cut(s["v"]))
        if s["case"]["bits"] == 8:
            views.update(m_scale=cut_top(s["ms"]), v_scale=cut_top(s["vs"]))
        if "copy" in s:
            views.update(copies=cut(s["copy"]))
        s["tensors"] = rgnn.AdamwTensors(**views)
    rgnn.adamw_step(s["tensors"], step=s["step"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY)


def _adamw(s):
    s["step"] += 1
    if own:
        _adamw_own(s)
    else:
        _adamw_plain(s)
    out = {"p": s["p"], "m": s["m"], "v": s["v"]}
    if s["case"]["bits"] == 8:
        # the values that the 8-bit states stand for: the scales in 32 bits, the codes' part as 16-bit values
        out.update(m=_decode_m(s["m"], torch.ones_like(s["ms"])).bfloat16(), ms=s["ms"],
                   v=_decode_v(s["v"], torch.ones_like(s["vs"])).bfloat16(), vs=s["vs"])
    if "copy" in s:
        out["copy"] = s["copy"]
    return out


def _linear_own(s):
    from paper_2301_06284_amd import rgnn
    c, x = s["case"], s["x"]
    y = torch.empty(c["M"], c["N"], dtype=x.dtype, device=x.device)
    out = {"y": y}
    if c["op"].startswith("fp8"):
        if c["op"] == "fp8_new":
            wq, ws = rgnn.fp8_quantize_weights(s["w"])
            out.update(wq=wq, ws=ws)
        else:
            wq, ws = s["wq"], s["ws"]
        xq, xs = rgnn.fp8_quantize_rows(x)
        out.update(xq=xq, xs=xs)
        rgnn.typed_linear_fp8(xq, xs, s["ptr"], wq, ws, y, gather=s["gather"], scatter=s["scatter"])
        return out
    rgnn.typed_linear(x, s["ptr"], s["w"], y, gather=s["gather"], scatter=s["scatter"])
    if c["op"] == "step":
        out["dx"], out["dw"] = torch.empty_like(x), torch.empty_like(s["w"])
        if "work" not in s:
            n = rgnn.typed_linear_wgrad_workspace_size(x.dtype, c["M"], c["T"], c["K"], c["N"])
            s["work"] = torch.empty(n, dtype=torch.uint8, device=x.device)
        rgnn.typed_linear(s["dy"], s["ptr"], s["w"], out["dx"], trans_w=True)
        rgnn.typed_linear_wgrad(x, s["dy"], s["ptr"], out["dw"], s["work"])
    return out


def _linear_plain(s):
    c, ptr, dt = s["case"], s["host_ptr"], s["x"].dtype
    if c["op"].startswith("fp8"):
        wq, ws = _quantize_weights(s["w"]) if c["op"] == "fp8_new" else (s["wq"], s["ws"])
        xq, xs = _quantize_rows(s["x"])
        x = _read_rows(xq, xs)
        x = x if s["gather"] is None else x[s["gather"].long()]
        out = {"y": _place(s, _products(ptr, x, _read_weights(wq, ws)), dt), "xq": xq, "xs": xs}
        return dict(out, wq=wq, ws=ws) if c["op"] == "fp8_new" else out
    x, w = _rows(s), s["w"].float()
    out = {"y": _place(s, _products(ptr, x, w), dt)}
    if c["op"] == "step":
        dy = s["dy"].float()
        out["dx"] = _products(ptr, dy, w.transpose(1, 2)).to(dt)
        out["dw"] = _outer(ptr, x, dy, c["T"]).to(dt)
    return out


def run(state):
    if state["case"]["op"] == "adamw":
        return _adamw(state)
    return _linear_own(state) if own else _linear_plain(state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "adamw":
        n = sum(_tensor_sizes(case))
        state = 16 if case["bits"] == 32 else 4 + 16 / QBLOCK
        per = 2 * SIZE[case["dtype"]] + SIZE[case["grad"]] + state + (2 if case["copy"] else 0)
        return {"bytes": n * per, "flops": n * 15}
    m, k, n, el = case["M"], case["K"], case["N"], SIZE[case["dtype"]]
    sizes = _sizes(case)
    weights = int((sizes > 0).sum()) * k * n
    flops = 2.0 * m * k * n
    if case["op"].startswith("fp8"):
        moved = case["X"] * k * el + case["X"] * (_kp(k) + _ks(k)) + m * n * el + weights * (1 + 1 / BLOCK ** 2)
        if case["op"] == "fp8_new":   # every weight is read and its codes written
            moved += case["T"] * k * n * (el + 1)
        return {"bytes": moved, "flops": flops}
    moved = min(case["X"], m) * k * el + m * n * el + weights * el + (8 * m if case["index"] else 0)
    if case["op"] == "step":   # the output gradient read, the input's and the weights' written
        return {"bytes": moved + m * (n + k) * el + case["T"] * k * n * el, "flops": 3 * flops}
    return {"bytes": moved, "flops": flops}


# ------------------------------------------------------------------ 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s)
    ptr, x = s["host_ptr"], s["x"].double()
    out = {}
    if case["op"].startswith("fp8"):
        x = _round_blocks(x, 1)
        w = _round_blocks(s["w"].double().transpose(1, 2), BLOCK) if case["op"] == "fp8_new" else \
            s["wq"].double() * torch.ldexp(torch.ones((), dtype=torch.float64, device="cuda"), s["ws"].int() - 127) \
            .repeat_interleave(BLOCK, 1)[:, :case["N"]].repeat_interleave(BLOCK, 2)[:, :, :_kp(case["K"])]
        w = w.transpose(1, 2)[:, :case["K"]]
    else:
        w = s["w"].double()
    rows = x if s["gather"] is None else x.index_select(0, s["gather"])
    y = torch.zeros(case["M"], case["N"], dtype=torch.float64, device="cuda")
    place = torch.arange(case["M"], device="cuda") if s["scatter"] is None else s["scatter"].long()
    dx, dw = torch.zeros_like(rows), torch.zeros(case["T"], case["K"], case["N"], dtype=torch.float64, device="cuda")
    for t, (a, b) in enumerate(zip(ptr, ptr[1:])):
        y.index_copy_(0, place[a:b], rows[a:b] @ w[t])
        if case["op"] == "step":
            d = s["dy"][a:b].double()
            dx[a:b], dw[t] = d @ w[t].t(), rows[a:b].t() @ d
    out["y"] = y
    if case["op"] == "step":
        out.update(dx=dx, dw=dw)
    return out


def _round_blocks(x, tall):
    """x [..., R, K] in 64 bits, each block of `tall` x 128 rounded to e4m3 under its own power of two."""
    r, k = x.shape[-2:]
    p = torch.nn.functional.pad(x, (0, -k % BLOCK, 0, -r % tall))
    b = p.unflatten(-1, (-1, BLOCK)).unflatten(-3, (-1, tall))
    top = b.abs().amax(dim=(-1, -3), keepdim=True)
    f, e = torch.frexp(top / 448)               # top / 448 = f 2^e with f in [1/2, 1)
    e = torch.where(f == 0.5, e - 1, e).clamp(min=-126)
    e = torch.where(top > 0, e, torch.zeros_like(e))
    v = torch.ldexp(b, -e)
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v)[1].clamp(min=-5) - 4)   # 3 bits behind the leading one
    v = torch.ldexp(torch.round(v / step) * step, e)
    return v.flatten(-4, -3).flatten(-2, -1)[..., :r, :k]


def _exact_adamw(s):
    eight, t = s["case"]["bits"] == 8, s["step"] + 1
    g, p = s["grad"].double(), s["p"].double()
    if eight:
        m, v = _decode_m(s["m"], s["ms"].double()), _decode_v(s["v"], s["vs"].double())
    else:
        m, v = s["m"].double(), s["v"].double()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    out = {"p": p, "m": m, "v": v}
    if eight:
        mb, vb = m.view(-1, QBLOCK), v.view(-1, QBLOCK)
        ms, vs = mb.abs().amax(dim=1), vb.amax(dim=1)
        cm = torch.round(127 * (mb.abs() / ms[:, None].clamp(min=1e-300)).sqrt()) / 127
        cv = torch.round(255 * (vb / vs[:, None].clamp(min=1e-300)) ** 0.25).clamp(min=1) * (vb > 0) / 255
        out.update(m=(cm * cm * torch.sign(mb)).view(-1), ms=ms, v=(cv ** 4).view(-1), vs=vs)
    if "copy" in s:
        out["copy"] = p
    return out
