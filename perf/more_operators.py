"""Performance cases of what stands between a layer's products: the root-mean-square
norm with the residual's addition, its backward pass and its outputs in 8 bits, dropout
from a counter-based generator whose mask is never stored, and the typed linear in 8-bit
integers with a scale for each row and each channel.

A case names an operation (`op`):

  norm          r = residual + D(x), y = r / rms(r) * w, as rows or as 8-bit codes with scales
  norm_step     the same with its gradients of x, of the residual and of w
  dropout       y = residual + D(x)
  dropout_step  the same with its gradient
  int8          rows quantised to 8-bit integers, then the product with weights kept so
  int8_new      the same with the weights quantised in the pass too (new weights)
  serve         norm straight into 8-bit integers, then the product that reads them

D keeps a value where a 32-bit number of its own is at least floor(p 2^32), times the 32-bit number
nearest to 1 / (1 - p), and makes it zero elsewhere.  The number of row i, column j is word j % 4 of Philox4x32-10 (Salmon et al.,
"Parallel random numbers: as easy as 1, 2, 3", 2011) for the counter (j / 4, i, o, o >> 32) and
the key (seed, seed >> 32), with rng = (seed, offset) on the device and o = offset + the call's number.

`run` computes them in elementary torch operations in 32 bits (what lies next to the border of a
code or of a 16-bit sum, and the generator's products, in 64), or (where `own`) with the calls of
paper_2301_06284_amd.rgnn.
"""
import math

import numpy as np
import torch

own = False

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2, "e4m3": 1}
BLOCK = 128       # codes lie in rows of whole blocks; elements of one e4m3 scale
EPS = 1e-6
CALL = 3          # the dropout's number among the calls of a step
LEAST = 2.0 ** -126


def listed():
    norm = dict(op="norm", x="bf16", res="bf16", w="bf16", y="bf16", rows=8, cols=2048, pad=0, p=0.0)
    drop = dict(op="dropout", x="bf16", res="", rows=292, cols=64, pad=0, p=0.1)
    int8 = dict(op="int8", x="bf16", M=16, X=8, T=32, K=2048, N=1536, skew=0.0, index=True)
    return [
        # serving, single tokens: latency
        dict(norm, name="norm_tokens"),
        # a graph layer's node features in fp32: short rows, many of them
        dict(norm, name="norm_nodes", x="fp32", res="fp32", w="fp32", y="fp32", rows=1000003, cols=64),
        # a long prompt in front of the 8-bit typed linear: codes and block scales
        dict(norm, name="norm_prompt_e4m3", y="e4m3", rows=8192, cols=4096),
        # a training step: dropout, the residual kept in fp32
        dict(norm, name="norm_step_wide", op="norm_step", res="fp32", w="fp32", rows=16384, cols=2048, p=0.1),
        # a training step in fp16 with a width that fills no vector
        dict(norm, name="norm_step_odd", op="norm_step", x="fp16", res="fp16", w="fp32", y="fp16", rows=10007, cols=333),
        # a mini-batch of sampled nodes in fp32: latency
        dict(drop, name="dropout_batch", x="fp32"),
        # a training step of a long batch, with the residual's addition
        dict(drop, name="dropout_step_wide", op="dropout_step", res="bf16", rows=16384, cols=4096),
        # columns cut out of a wider matrix, of an odd width
        dict(drop, name="dropout_cut", x="fp16", rows=300007, cols=77, pad=24, p=0.5),
        # serving, single tokens: 8 tokens, two of 32 weights each; the weights' bytes
        dict(int8, name="int8_tokens"),
        # one dense weight, a long prompt: the matrix cores
        dict(int8, name="int8_dense", M=8192, X=8192, T=1, K=4096, N=4096, index=False),
        # after an update of the weights: they are quantised again, then used
        dict(int8, name="int8_new_weights", op="int8_new", M=4099, X=4099, T=16, skew=0.4, index=False),
        # serving a batch: norm, codes, product
        dict(int8, name="serve_batch", op="serve", res="bf16", M=2050, X=2050, T=16, K=1536, N=2048, skew=0.4, index=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A feature width: mostly whole vectors of 16 bytes, one in four any number."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.25 else max(8, w // 8 * 8)


def draw(rng):
    op = rng.choice(["norm", "norm", "norm", "norm_step", "norm_step", "dropout", "dropout_step", "int8", "int8_new", "serve"])
    x = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op in ("int8", "int8_new", "serve"):
        t = _log_int(rng, 1, 32)
        m, k, n = _log_int(rng, 1, 8192), _width(rng, 64, 3000), _width(rng, 64, 3000)
        index = op != "serve" and rng.random() < 0.5
        rows = max(1, int(m * rng.uniform(0.4, 1.2))) if index else m
        c = dict(op=op, x=x, M=m, X=rows, T=t, K=k, N=n, skew=round(rng.uniform(0.0, 0.6), 2), index=index)
        if op == "serve":
            x = "bf16" if x == "fp32" else x
            c.update(x=x, res=rng.choice(["", x]))
        return c
    cols = _width(rng, 16, 10000)
    rows = _log_int(rng, 1, max(2, min(600000, 30000000 // cols)))
    pad = rng.choice([0, 0, 0, 8, 24, 7])
    res = rng.choice(["", x, "fp32"])
    p = rng.choice([0.0, 0.1, 0.5]) if op.startswith("norm") else rng.choice([0.05, 0.1, 0.5])
    c = dict(op=op, x=x, res=res, rows=rows, cols=cols, pad=pad, p=p)
    if op.startswith("norm"):
        c.update(w=rng.choice([x, "fp32"]), y=rng.choice([x, x, "e4m3"]) if op == "norm" else x)
    return c


# ------------------------------------------------------------------ inputs

def _sizes(case):
    """Rows of each type: a multinomial draw of Zipf shares, the same for every seed."""
    r = np.random.RandomState(11 + case["M"] + 13 * case["T"])
    p = 1.0 / np.arange(1, case["T"] + 1) ** case["skew"]
    r.shuffle(p)
    return r.multinomial(case["M"], p / p.sum())


def _kp(k):
    return -(-k // BLOCK) * BLOCK


def _ks(k):
    return -(-k // (4 * BLOCK)) * 4


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731

    def rows_of(rows, cols, pad, dt):
        """Rows of very different size, as activations have, some of them zero, as those of nodes without edges are."""
        m = randn(rows, cols + pad) * torch.exp(randn(rows, 1))
        m[5::97] = 0
        return m.to(DT[dt])[:, :cols]

    s = dict(case=case)
    if "T" in case:
        t, k, n = case["T"], case["K"], case["N"]
        ptr = np.concatenate([[0], np.cumsum(_sizes(case))]).astype(np.int64)
        s.update(x=rows_of(case["X"], k, 0, case["x"]), host_ptr=ptr.tolist(), ptr=torch.from_numpy(ptr).cuda(),
                 gather=None, scatter=None)
        w = randn(t, k, n).mul_(1.0 / math.sqrt(k)).to(DT[case["x"]])
        if case["index"]:
            s["gather"] = torch.randint(0, case["X"], (case["M"],), generator=g, device="cuda", dtype=torch.int32)
            s["scatter"] = torch.randperm(case["M"], generator=g, device="cuda").to(torch.int32)
        if case["op"] == "int8_new":
            s["w"] = w
        else:
            s["wq"], s["ws"] = _int8_weights(w)
        if case["op"] == "serve":
            s["weight"] = (1 + 0.1 * randn(k)).to(DT[case["x"]])
            s["res"] = rows_of(case["X"], k, 0, case["res"]) if case["res"] else None
        return s
    rows, cols, pad = case["rows"], case["cols"], case["pad"]
    s["x"] = rows_of(rows, cols, pad, case["x"])
    s["res"] = rows_of(rows, cols, 0, case["res"]) if case["res"] else None
    s["rng"] = torch.tensor([seed * 0x9E3779B97F4A7C15 % 2 ** 63, 1000 + seed], dtype=torch.int64, device="cuda")
    if case["op"].startswith("norm"):
        s["weight"] = (1 + 0.1 * randn(cols)).to(DT[case["w"]])
    if case["op"].endswith("step"):
        s["dy"] = (randn(rows, cols) * 0.01).to(DT[case["y"] if "y" in case else case["res"] or case["x"]])
        if case["op"] == "norm_step" and case["res"]:     # the gradient that arrives along the residual
            s["dsum"] = (randn(rows, cols) * 0.01).to(DT[case["res"]])
    return s


# ------------------------------------------------------------------ plain forms

def _philox(rows, cols, rng, call):
    """The 32-bit numbers of a matrix, as int64 [rows, cols]: products of 32 bits in 64, whose
    upper half a shift brings down and a mask frees of the sign."""
    low = 0xFFFFFFFF
    off = rng[1] + call
    c0 = torch.arange(-(-cols // 4), device="cuda").expand(rows, -1)
    c1 = torch.arange(rows, device="cuda")[:, None].expand_as(c0)
    c2, c3 = (off & low).expand_as(c0), (off >> 32 & low).expand_as(c0)
    k0, k1 = rng[0] & low, rng[0] >> 32 & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack([c0, c1, c2, c3], dim=2).view(rows, -1)[:, :cols]


def _keep(s):
    return _philox(s["case"]["rows"], s["case"]["cols"], s["rng"], CALL) >= math.floor(s["case"]["p"] * 2.0 ** 32)


def _factor(s):
    return float(np.float32(1.0 / (1.0 - s["case"]["p"])))


def _drop(s, x, keep):
    return x if keep is None else torch.where(keep, x * _factor(s), torch.zeros_like(x))


def _scale_bytes(top):
    """The biased exponent of the least power of two s with top <= 448 s (at least 2^-126),
    from the bits of the largest magnitude `top` (fp32)."""
    bits = top.view(torch.int32)
    return (((bits + 0x1FFFFF) >> 23) - 8).clamp(1, 254)


def _e4m3_rows(x):
    """[rows, K] -> codes [rows, Kp] and scale bytes [rows, Ks] (127, a scale of 1, behind the last block)."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x, (0, _kp(k) - k)).view(rows, -1, BLOCK)
    e = _scale_bytes(x.abs().amax(dim=2))
    q = (x * torch.exp2((127 - e).float()).unsqueeze(2)).view(rows, -1).to(torch.float8_e4m3fn)
    return q, torch.nn.functional.pad(e, (0, _ks(k) - e.shape[1]), value=127).to(torch.uint8)


def _int8(x, dim):
    """Codes of x (32 bits) and their scales along `dim`: x times the 32-bit inverse of the scale, rounded once.
    (The quotient in 64 bits: in 32, torch multiplies by the rounded inverse of 127.)"""
    scale = (x.abs().amax(dim=dim, keepdim=True).double() / 127.0).float().clamp(min=LEAST)
    return torch.round(x.double() * (1.0 / scale).double()).to(torch.int8), scale


def _int8_rows(x):
    """[rows, K] -> codes [rows, Kp], zero behind K, and scales [rows]."""
    q, scale = _int8(x.float(), 1)
    return torch.nn.functional.pad(q, (0, _kp(x.shape[1]) - x.shape[1])), scale.view(-1)


def _int8_weights(w):
    """[T, K, N] -> codes [T, N, Kp] and scales [T, N], one for each channel."""
    q, scale = _int8(w.float(), 1)
    return torch.nn.functional.pad(q.transpose(1, 2), (0, _kp(w.shape[1]) - w.shape[1])).contiguous(), scale[:, 0].contiguous()


def _norm(s, keep, y):
    """(r rounded to its type, y in 32 bits, 1 / rms)."""
    wide = torch.float32 if keep is None else torch.float64     # a 24-bit factor's product, rounded with the sum
    r = _drop(s, s["x"].to(wide), keep)
    r = (r if s["res"] is None else s["res"].to(wide) + r).float().to(s["x"].dtype if s["res"] is None else s["res"].dtype)
    f = r.float()
    if y in ("e4m3", "int8"):       # codes: values next to a border
        rstd = (1.0 / torch.sqrt(f.double().square().mean(dim=1, keepdim=True) + EPS)).float()
    else:
        rstd = 1.0 / torch.sqrt(f.square().mean(dim=1, keepdim=True) + EPS)
    return r, f * rstd * s["weight"].float(), rstd


def _norm_plain(s):
    c = s["case"]
    keep = _keep(s) if c["p"] else None
    r, y, rstd = _norm(s, keep, c["y"])
    out = {"sum": r} if c["res"] or c["p"] else {}
    if c["y"] == "e4m3":
        out["y"], out["scales"] = _e4m3_rows(y)
    else:
        out["y"] = y.to(DT[c["y"]])
    if c["op"] == "norm_step":
        w, dy = s["weight"].float(), s["dy"].float()
        n, g = r.float() * rstd, dy * w
        dr = rstd * (g - n * (g * n).mean(dim=1, keepdim=True))
        if "dsum" in s:
            dr = dr + s["dsum"].float()
        if c["res"]:
            out["dres"] = dr.to(DT[c["res"]])
        if c["p"] or c["res"] != c["x"]:
            out["dx"] = _drop(s, dr, keep).to(DT[c["x"]])
        out["dw"] = (dy * n).sum(dim=0).to(s["weight"].dtype)
    return out


def _norm_own(s):
    from paper_2301_06284_amd import rgnn
    c, x = s["case"], s["x"]
    rows, cols = x.shape
    drop = None
    if c["p"]:
        if "drop" not in s:
            s["drop"] = rgnn.Dropout(c["p"], s["rng"], CALL)
        drop = s["drop"]
    out, scales, rstd, total = {}, None, None, None
    if c["res"] or c["p"]:
        out["sum"] = total = torch.empty(rows, cols, dtype=DT[c["res"] or c["x"]], device=x.device)
    if c["y"] == "e4m3":
        out["y"] = torch.empty(rows, _kp(cols), dtype=torch.float8_e4m3fn, device=x.device)
        out["scales"] = scales = torch.empty(rows, _ks(cols), dtype=torch.uint8, device=x.device)
    else:
        out["y"] = torch.empty(rows, cols, dtype=DT[c["y"]], device=x.device)
    step = c["op"] == "norm_step"
    if step:
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    rgnn.rms_norm(x, s["weight"], out["y"], eps=EPS, residual=s["res"], sum=total, scales=scales, rstd=rstd, dropout=drop)
    if step:
        if "work" not in s:
            s["work"] = torch.empty(rgnn.rms_norm_backward_workspace_size(rows, cols), dtype=torch.uint8, device=x.device)
        if c["res"]:
            out["dres"] = torch.empty(rows, cols, dtype=DT[c["res"]], device=x.device)
        if c["p"] or c["res"] != c["x"]:
            out["dx"] = torch.empty(rows, cols, dtype=x.dtype, device=x.device)
        out["dw"] = torch.empty_like(s["weight"])
        rgnn.rms_norm_backward(s["dy"], x if total is None else total, rstd, s["weight"], d_sum=s.get("dsum"),
                               d_residual=out.get("dres"), dX=out.get("dx"), dW=out["dw"], ws=s["work"], dropout=drop)
    return out


def _dropout_plain(s):
    c, keep = s["case"], _keep(s)
    y = _drop(s, s["x"].float(), keep)
    y = y if s["res"] is None else s["res"].float() + y
    out = {"y": y.to(DT[c["res"] or c["x"]])}
    if c["op"] == "dropout_step":
        out["dx"] = _drop(s, s["dy"].float(), keep).to(s["x"].dtype)
    return out


def _dropout_own(s):
    from paper_2301_06284_amd import rgnn
    c, x = s["case"], s["x"]
    if "drop" not in s:
        s["drop"] = rgnn.Dropout(c["p"], s["rng"], CALL)
    out = {"y": torch.empty(x.shape, dtype=DT[c["res"] or c["x"]], device=x.device)}
    rgnn.dropout(x, out["y"], s["drop"], residual=s["res"])
    if c["op"] == "dropout_step":
        out["dx"] = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rgnn.dropout(s["dy"], out["dx"], s["drop"])
    return out


def _linear_plain(s):
    c, out = s["case"], {}
    if c["op"] == "int8_new":
        wq, ws = out["wq"], out["ws"] = _int8_weights(s["w"])
    else:
        wq, ws = s["wq"], s["ws"]
    if c["op"] == "serve":
        out["sum"], y, _ = _norm(s, None, "int8")
        if s["res"] is None:
            del out["sum"]
        xq, xs = _int8_rows(y)
    else:
        xq, xs = _int8_rows(s["x"])
    x = xq.float()
    scale = xs
    if s["gather"] is not None:
        x, scale = x[s["gather"].long()], xs[s["gather"].long()]
    y = torch.empty(c["M"], c["N"], device="cuda")
    ptr = s["host_ptr"]
    for t in range(c["T"]):
        a, b = ptr[t], ptr[t + 1]
        if b > a:
            y[a:b] = (x[a:b] @ wq[t].float().t()) * scale[a:b, None] * ws[t]
    if s["scatter"] is not None:
        y[s["scatter"].long()] = y.clone()
    # codes are whole numbers and come as such beside their scales
    return dict(out, y=y.to(s["x"].dtype), xq=xq, xs=xs)


def _linear_own(s):
    from paper_2301_06284_amd import rgnn
    c, x = s["case"], s["x"]
    out = {"y": torch.empty(c["M"], c["N"], dtype=x.dtype, device=x.device)}
    if c["op"] == "int8_new":
        wq, ws = out["wq"], out["ws"] = rgnn.int8_quantize_weights(s["w"])
    else:
        wq, ws = s["wq"], s["ws"]
    if c["op"] == "serve":
        xq = torch.empty(c["X"], _kp(c["K"]), dtype=torch.int8, device=x.device)
        xs = torch.empty(c["X"], dtype=torch.float32, device=x.device)
        total = None
        if c["res"]:
            out["sum"] = total = torch.empty(c["X"], c["K"], dtype=DT[c["res"]], device=x.device)
        rgnn.rms_norm(x, s["weight"], xq, eps=EPS, residual=s["res"], sum=total, scales=xs)
    else:
        xq, xs = rgnn.int8_quantize_rows(x)
    rgnn.typed_linear_int8(xq, xs, s["ptr"], wq, ws, out["y"], gather=s["gather"], scatter=s["scatter"])
    return dict(out, xq=xq, xs=xs)


def run(state):
    op = state["case"]["op"]
    if op.startswith("norm"):
        return _norm_own(state) if own else _norm_plain(state)
    if op.startswith("dropout"):
        return _dropout_own(state) if own else _dropout_plain(state)
    return _linear_own(state) if own else _linear_plain(state)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    x = SIZE[case["x"]]
    res = SIZE[case["res"]] if case.get("res") else 0
    if "T" in case:
        m, k, n = case["M"], case["K"], case["N"]
        weights = int((_sizes(case) > 0).sum()) * k * n
        moved = case["X"] * (k * (x + 1) + 4) + m * n * x + weights + (8 * m if case["index"] else 0)
        if case["op"] == "int8_new":   # every weight is read and its codes written
            moved += case["T"] * k * n * (x + 1) + case["T"] * n * 4
        if case["op"] == "serve":      # the residual read, the sum written
            moved += case["X"] * k * 2 * res + k * x
        return {"bytes": moved, "flops": 2.0 * m * k * n + 8.0 * case["X"] * k}
    n, cols = case["rows"] * case["cols"], case["cols"]
    if case["op"].startswith("dropout"):
        step = case["op"] == "dropout_step"
        per = x + res + (res or x) + (x + (res or x) if step else 0)
        return {"bytes": n * per, "flops": n * (20.0 if step else 10.0)}
    per = x + res + SIZE[case["y"]] + ((res or x) if res or case["p"] else 0) + (1 / BLOCK if case["y"] == "e4m3" else 0)
    moved = n * per + cols * SIZE[case["w"]]
    if case["op"] == "norm_step":
        moved += n * (SIZE[case["y"]] + 2 * res + (x if case["p"] or case["res"] != case["x"] else 0)) + cols * SIZE[case["w"]]
    return {"bytes": moved, "flops": n * (24.0 if case["op"] == "norm_step" else 8.0)}


# ------------------------------------------------------------------ 64 bits, from the definitions

def _words(rows, cols, seed, offset):
    """The generator once more, on 16-bit limbs: [rows, cols] of its numbers."""
    def product(a, b):     # of 32-bit a (tensor) and b: (upper, lower 32 bits)
        ah, al, bh, bl = a >> 16, a & 0xFFFF, b >> 16, b & 0xFFFF
        mid = ah * bl + (al * bl >> 16)
        cross = al * bh + (mid & 0xFFFF)
        return ah * bh + (mid >> 16) + (cross >> 16), (cross & 0xFFFF) << 16 | al * bl & 0xFFFF
    words = []
    col, row = torch.meshgrid(torch.arange(-(-cols // 4), device="cuda"), torch.arange(rows, device="cuda"), indexing="xy")
    x = [col, row, torch.full_like(col, offset % 2 ** 32), torch.full_like(col, offset // 2 ** 32 % 2 ** 32)]
    for i in range(10):
        key = (seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32
        (h0, l0), (h2, l2) = product(x[0], 0xD2511F53), product(x[2], 0xCD9E8D57)
        x = [h2 ^ x[1] ^ key[0], l2, h0 ^ x[3] ^ key[1], l0]
    words = torch.zeros(rows, x[0].shape[1] * 4, dtype=torch.int64, device="cuda")
    for q in range(4):
        words[:, q::4] = x[q]
    return words[:, :cols]


def _exact_drop(s, v):
    p = s["case"].get("p", 0.0)
    if not p:
        return v
    seed, offset = s["rng"].tolist()
    if "kept" not in s:
        s["kept"] = _words(*v.shape, seed, offset + CALL) >= int(p * 2 ** 32)
    return (v * np.float64(np.float32(1 / (1 - p)))).masked_fill(~s["kept"], 0.0)


def _exact_int8(x):
    """(codes, scale) of rows of x; the scale and its inverse are numbers of 32 bits by definition."""
    scale = torch.maximum((x.abs().max(dim=-1).values / 127).float(), torch.full((), LEAST, device=x.device))
    return torch.round(x * scale.reciprocal().double()[..., None]), scale.double()


def _exact_e4m3(x):
    """Codes as numbers, of blocks of a row under their own power of two."""
    k = x.shape[1]
    b = torch.nn.functional.pad(x, (0, -k % BLOCK)).unflatten(1, (-1, BLOCK))
    top = b.abs().amax(dim=2, keepdim=True)
    f, e = torch.frexp(top / 448)               # top / 448 = f 2^e with f in [1/2, 1)
    e = torch.where(f == 0.5, e - 1, e).clamp(min=-126)
    v = torch.ldexp(b, torch.where(top > 0, -e, torch.zeros_like(e)))
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v)[1].clamp(min=-5) - 4)   # 3 bits behind the leading one
    return (torch.round(v / step) * step).flatten(1)


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["op"].startswith("dropout"):
        y = _exact_drop(s, x)
        out = {"y": y if s["res"] is None else y + s["res"].double()}
        if case["op"] == "dropout_step":
            out["dx"] = _exact_drop(s, s["dy"].double())
        return out
    out = {}
    if case["op"].startswith("norm") or case["op"] == "serve":
        r = _exact_drop(s, x)
        if s["res"] is not None:
            r = r + s["res"].double()
        if case["res"] or case.get("p"):
            out["sum"] = r
        r = r.to(DT[case["res"] or case["x"]]).double()      # y is of the sum as it is kept
        w = s["weight"].double()
        rms = torch.sqrt((r * r).mean(dim=1) + EPS)[:, None]
        y = r / rms * w
        if case["op"] == "serve":
            x = y
        else:
            out["y"] = _exact_e4m3(y) if case["y"] == "e4m3" else y
    if case["op"] == "norm_step":
        g, n = s["dy"].double() * w, r / rms
        dr = (g - n * (g * n).mean(dim=1)[:, None]) / rms
        if "dsum" in s:
            dr = dr + s["dsum"].double()
        if case["res"]:
            out["dres"] = dr
        if case["p"] or case["res"] != case["x"]:
            out["dx"] = _exact_drop(s, dr)
        out["dw"] = torch.einsum("ij,ij->j", s["dy"].double(), n)
    if "T" not in case:
        return out
    codes, out["xs"] = _exact_int8(x)
    if case["op"] == "int8_new":
        wcodes, out["ws"] = _exact_int8(s["w"].double().transpose(1, 2))
    else:
        wcodes, out["ws"] = s["wq"][:, :, :case["K"]].double(), s["ws"].double()
    rows = torch.arange(case["M"], device="cuda") if s["gather"] is None else s["gather"].long()
    place = torch.arange(case["M"], device="cuda") if s["scatter"] is None else s["scatter"].long()
    y = torch.zeros(case["M"], case["N"], dtype=torch.float64, device="cuda")
    for t, (a, b) in enumerate(zip(s["host_ptr"], s["host_ptr"][1:])):
        at = rows[a:b]
        y[place[a:b]] = (codes[at] @ wcodes[t].t()) * out["xs"][at][:, None] * out["ws"][t]
    out["y"] = y
    if case["op"] != "int8_new":
        del out["ws"]
    return out
