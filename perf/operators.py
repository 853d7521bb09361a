"""The operators around a projection GEMM in training, as measured cases.

A pre-norm projection block computes y = layer_norm(x), o = y . W and, going
back, dW = y^T . do and the layer norm's gradients.  Beside the GEMMs, which
the library has, that takes:

  ln_forward   layer norm of the rows of x, with the rows' mean and 1/std kept
               for the backward pass and, optionally, the result's 8-bit
               checkpoint written in the same pass;
  ln_backward  the gradients of x, gamma and beta, x being what the forward
               pass read or its 8-bit checkpoint;
  checkpoint   an activation saved in 8 bits and restored;
  weight_grad  dW = base + X^T . dY with X read from its 8-bit checkpoint.

The checkpoint holds blocks of 32 consecutive values of a row: a power of two
2^E, E the least exponent >= -126 with max|x| <= 127 * 2^E (one byte, E + 127;
255 for a block with a NaN or an infinity), and 32 signed bytes
round_half_even(x / 2^E).

``own`` selects between the plain form (elementary torch operations in 32
bits) and the library's calls.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
LARGEST_ELEMENTS = 8192 * 12288
LARGEST_MACS = 8192 * 4096 * 11008


def listed():
    return [
        # one decoding-sized batch of tokens through a 4096-wide layer norm: launch latency
        {"name": "ln fwd 16x4096", "op": "ln_forward", "rows": 16, "cols": 4096, "x": "bf16", "y": "bf16",
         "params": "bf16", "save": False, "pad": 0},
        # a training micro-batch; the result is also checkpointed for the weight gradient
        {"name": "ln fwd 8192x4096 saved", "op": "ln_forward", "rows": 8192, "cols": 4096, "x": "bf16", "y": "bf16",
         "params": "f32", "save": True, "pad": 0},
        # a float32 residual stream of an odd width, rows not 16-byte aligned
        {"name": "ln fwd 2560x777 f32", "op": "ln_forward", "rows": 2560, "cols": 777, "x": "f32", "y": "bf16",
         "params": "f32", "save": False, "pad": 0},
        # backward of a short micro-batch
        {"name": "ln bwd 2048x4096", "op": "ln_backward", "rows": 2048, "cols": 4096, "x": "bf16", "dy": "bf16",
         "params": "bf16", "from8": False, "pad": 0},
        # backward of a wide layer over a full micro-batch: memory-bound
        {"name": "ln bwd 8192x12288", "op": "ln_backward", "rows": 8192, "cols": 12288, "x": "bf16", "dy": "bf16",
         "params": "f32", "from8": False, "pad": 0},
        # x restored from its 8-bit checkpoint on the way, float32 gradient of the residual stream,
        # rows that are a slice of a wider buffer
        {"name": "ln bwd 1000x1500 from 8 bits", "op": "ln_backward", "rows": 1000, "cols": 1500, "x": "f32",
         "dy": "bf16", "params": "f32", "from8": True, "pad": 36},
        # a small activation: latency
        {"name": "checkpoint 128x4096", "op": "checkpoint", "rows": 128, "cols": 4096, "x": "bf16", "pad": 0},
        # a feed-forward activation of a full micro-batch: memory-bound
        {"name": "checkpoint 8192x11008", "op": "checkpoint", "rows": 8192, "cols": 11008, "x": "bf16", "pad": 0},
        # few tokens, gradient added to the float32 one of earlier micro-batches: bound by dW
        {"name": "weight grad 128t 4096x4096", "op": "weight_grad", "tokens": 128, "k": 4096, "n": 4096, "w": "f32",
         "layout": "KxN", "base": True},
        # a short micro-batch, square projection, bf16 gradient in the layout of a column-major weight
        {"name": "weight grad 2048t 4096x4096", "op": "weight_grad", "tokens": 2048, "k": 4096, "n": 4096,
         "w": "bf16", "layout": "NxK", "base": False},
        # odd sizes: no operand row 16-byte aligned
        {"name": "weight grad 1000t 777x1501", "op": "weight_grad", "tokens": 1000, "k": 777, "n": 1501, "w": "f32",
         "layout": "KxN", "base": False},
        # a full micro-batch of a feed-forward projection: bound by the tensor cores
        {"name": "weight grad 8192t 4096x11008", "op": "weight_grad", "tokens": 8192, "k": 4096, "n": 11008,
         "w": "f32", "layout": "KxN", "base": False},
    ]


def _size(rng, lo, hi, step=8):
    """A size between lo and hi, spread over its logarithm; two in three a multiple of `step`, else any."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 2 / 3 and v > step:
        v = v // step * step
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["ln_forward", "ln_backward", "checkpoint", "weight_grad"])
    if op == "weight_grad":
        while True:
            t, k, n = _size(rng, 1, 8192), _size(rng, 64, 11008), _size(rng, 64, 11008)
            if t * k * n <= LARGEST_MACS:
                break
        return {"op": op, "tokens": t, "k": k, "n": n, "w": rng.choice(["f32", "bf16"]),
                "layout": rng.choice(["KxN", "NxK"]), "base": rng.random() < 0.5}
    while True:
        rows, cols = _size(rng, 1, 16384), _size(rng, 64, 12288)
        if rows * cols <= LARGEST_ELEMENTS:
            break
    case = {"op": op, "rows": rows, "cols": cols, "x": rng.choice(["bf16", "f32"]),
            "pad": rng.choice([0, 0, 0, 8, 32, 5])}
    if op == "ln_forward":
        case.update(y=rng.choice(["bf16", "f32"]), params=rng.choice(["bf16", "f32"]), save=rng.random() < 0.5)
    elif op == "ln_backward":
        case.update(dy=rng.choice(["bf16", "f32"]), params=rng.choice(["bf16", "f32"]), from8=rng.random() < 0.3)
    return case


# ------------------------------------------------------------------- inputs

def _rows(shape, pad, dtype, fill):
    """A rows x cols matrix that is the left part of a buffer `pad` columns wider."""
    rows, cols = shape
    buf = torch.zeros((rows, cols + pad), dtype=dtype, device="cuda")
    if fill is not None:
        buf[:, :cols].copy_(fill)
    return buf[:, :cols]


def _activations(gen, rows, cols):
    """Activations as a transformer has them: channels of different scale and offset, one in a hundred an outlier
    channel, rows of different magnitude."""
    r = dict(generator=gen, device="cuda", dtype=torch.float32)
    x = torch.randn((rows, cols), **r)
    channel = torch.exp(0.4 * torch.randn(cols, **r))
    channel = torch.where(torch.rand(cols, **r) < 0.01, channel * 16, channel)
    return (x * channel + 0.2 * torch.randn(cols, **r)) * torch.exp(0.3 * torch.randn((rows, 1), **r))


def _params(gen, cols, dtype):
    r = dict(generator=gen, device="cuda", dtype=torch.float32)
    return (1 + 0.1 * torch.randn(cols, **r)).to(dtype), (0.1 * torch.randn(cols, **r)).to(dtype)


def _gradients(gen, rows, cols):
    """Gradients of small magnitude; one row in sixteen is a masked token's, all zero."""
    r = dict(generator=gen, device="cuda", dtype=torch.float32)
    g = 1e-3 * torch.randn((rows, cols), **r)
    return torch.where(torch.rand((rows, 1), **r) < 1 / 16, torch.zeros_like(g), g)


def _empty8(rows, cols):
    blocks = -(-cols // BLOCK)
    return (torch.zeros((rows, cols), dtype=torch.int8, device="cuda"),
            torch.zeros((rows, blocks), dtype=torch.uint8, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    s = dict(case)
    op = case["op"]
    if op == "weight_grad":
        t, k, n = case["tokens"], case["k"], case["n"]
        s["q8"], s["e8"] = _encode(_activations(gen, t, k))
        s["grad"] = _gradients(gen, t, n).to(torch.bfloat16)
        shape = (k, n) if case["layout"] == "KxN" else (n, k)
        wt = DTYPES[case["w"]]
        old = None
        if case["base"]:
            old = (1e-2 * torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)).to(wt)
        s["old"] = old
        s["new"] = torch.zeros(shape, dtype=wt, device="cuda")
        return s
    rows, cols, pad = case["rows"], case["cols"], case["pad"]
    xt = DTYPES[case["x"]]
    acts = _activations(gen, rows, cols)
    s["inp"] = _rows((rows, cols), pad, xt, acts)
    s["q8"], s["e8"] = _empty8(rows, cols)
    if op == "checkpoint":
        s["out"] = _rows((rows, cols), pad, xt, None)
        return s
    s["gamma"], s["beta"] = _params(gen, cols, DTYPES[case["params"]])
    if op == "ln_forward":
        s["out"] = _rows((rows, cols), pad, DTYPES[case["y"]], None)
        s["mean"] = torch.zeros(rows, dtype=torch.float32, device="cuda")
        s["rstd"] = torch.zeros(rows, dtype=torch.float32, device="cuda")
        s["restored"] = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda") if case["save"] else None
        return s
    x32 = s["inp"].float()
    s["mean"] = x32.mean(1)
    s["rstd"] = torch.rsqrt((x32 - s["mean"][:, None]).square().mean(1) + EPS)
    if case["from8"]:
        s["q8"], s["e8"] = _encode(x32)
        s["inp"] = None
    s["grad"] = _rows((rows, cols), pad, DTYPES[case["dy"]], _gradients(gen, rows, cols))
    s["out"] = _rows((rows, cols), pad, xt, None)
    s["dgamma"] = torch.zeros(cols, dtype=torch.float32, device="cuda")
    s["dbeta"] = torch.zeros(cols, dtype=torch.float32, device="cuda")
    return s


# ---------------------------------------------------------------- plain form

def _pow2(exponent):
    """2^exponent as float32, -126 <= exponent <= 127."""
    return ((exponent + 127) << 23).view(torch.float32)


def _encode(x):
    """(signed bytes, block exponents) of the float32 matrix x."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    v = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    top = v.abs().amax(2)
    m, ex = torch.frexp(top)                          # top = m * 2^ex, 0.5 <= m < 1
    e = torch.where(m > 127 / 128, ex - 6, ex - 7).clamp(-126, 122).to(torch.int32)
    e = torch.where(torch.isfinite(top), e, torch.full_like(e, 0))
    q = torch.round(v * _pow2(-e)[:, :, None])
    q = torch.where(torch.isfinite(top)[:, :, None], q, torch.zeros_like(q))
    code = torch.where(torch.isfinite(top), e + 127, torch.full_like(e, 255))
    return q.view(rows, -1)[:, :cols].to(torch.int8).contiguous(), code.to(torch.uint8)


def _decode(q, code):
    """The float32 values that signed bytes and block exponents stand for."""
    rows, cols = q.shape
    e = code.to(torch.int32)
    scale = torch.where(e == 255, torch.full(e.shape, math.nan, device=e.device), _pow2(e.clamp(1, 249) - 127))
    return q.float() * scale.repeat_interleave(BLOCK, dim=1)[:, :cols]


def _plain(s):
    op = s["op"]
    if op == "weight_grad":
        x, g = _decode(s["q8"], s["e8"]), s["grad"].float()
        w = x.t() @ g if s["layout"] == "KxN" else g.t() @ x
        if s["old"] is not None:
            w = w + s["old"].float()
        return {"dw": w.to(s["new"].dtype)}
    if op == "checkpoint":
        return {"x": _decode(*_encode(s["inp"].float())).to(s["out"].dtype)}
    gamma, beta = s["gamma"].float(), s["beta"].float()
    if op == "ln_forward":
        x = s["inp"].float()
        mean = x.mean(1)
        d = x - mean[:, None]
        rstd = 1 / torch.sqrt(d.square().mean(1) + EPS)
        y = (d * rstd[:, None] * gamma + beta).to(s["out"].dtype)
        r = {"y": y, "mean": mean, "rstd": rstd}
        if s["save"]:
            r["saved"] = _decode(*_encode(y.float())).to(torch.bfloat16)
        return r
    x = s["inp"].float() if s["inp"] is not None else _decode(s["q8"], s["e8"])
    dy = s["grad"].float()
    xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * gamma
    dx = s["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return {"dx": dx.to(s["out"].dtype), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}


# ------------------------------------------------------------- library's calls

def _ours(s):
    from paper_2512_13282_gb300 import layer as L
    op = s["op"]
    ty = {torch.float32: L.GEMM_TYPE_F32, torch.bfloat16: L.GEMM_TYPE_BF16}
    q, e = s["q8"], s["e8"]
    if op == "weight_grad":
        new, old, grad = s["new"], s["old"], s["grad"]
        L.check(L.gemm_q8_weight_grad(
            s["tokens"], s["k"], s["n"], q, q.stride(0), e, e.stride(0), grad, grad.stride(0),
            old, new.stride(0), new, new.stride(0),
            L.GEMM_B_ROW_MAJOR_KxN if s["layout"] == "KxN" else L.GEMM_B_COL_MAJOR_NxK, ty[new.dtype]))
        return {"dw": new}
    rows, cols, out = s["rows"], s["cols"], s["out"]
    x = s["inp"]
    if op == "checkpoint":
        L.check(L.gemm_q8_save(rows, cols, x, x.stride(0), ty[x.dtype], q, q.stride(0), e, e.stride(0)))
        L.check(L.gemm_q8_restore(rows, cols, q, q.stride(0), e, e.stride(0), out, out.stride(0), ty[out.dtype]))
        return {"x": out}
    if op == "ln_forward":
        save = s["save"]
        L.check(L.gemm_layernorm_forward(
            rows, cols, x, x.stride(0), ty[x.dtype], s["gamma"], s["beta"], ty[s["gamma"].dtype], EPS,
            out, out.stride(0), ty[out.dtype], s["mean"], s["rstd"],
            q if save else None, q.stride(0), e if save else None, e.stride(0)))
        r = {"y": out, "mean": s["mean"], "rstd": s["rstd"]}
        if save:
            back = s["restored"]
            L.check(L.gemm_q8_restore(rows, cols, q, q.stride(0), e, e.stride(0), back, back.stride(0),
                                      ty[back.dtype]))
            r["saved"] = back
        return r
    grad = s["grad"]
    from8 = x is None
    L.check(L.gemm_layernorm_backward(
        rows, cols, x, 0 if from8 else x.stride(0), ty[out.dtype], q if from8 else None, q.stride(0),
        e if from8 else None, e.stride(0), s["gamma"], ty[s["gamma"].dtype], s["mean"], s["rstd"],
        grad, grad.stride(0), ty[grad.dtype], out, out.stride(0), ty[out.dtype], s["dgamma"], s["dbeta"]))
    return {"dx": out, "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def run(state):
    return _ours(state) if own else _plain(state)


# ------------------------------------------------------------------ cost

def work(case):
    op = case["op"]
    if op == "weight_grad":
        t, k, n, w = case["tokens"], case["k"], case["n"], BYTES[case["w"]]
        moved = t * (k + -(-k // BLOCK)) + 2 * t * n + w * k * n * (2 if case["base"] else 1)
        return {"bytes": moved, "flops": 2 * t * k * n}
    rows, cols = case["rows"], case["cols"]
    n, held = rows * cols, rows * (cols + -(-cols // BLOCK))
    if op == "checkpoint":
        # the activation read, its checkpoint written and read, the restored activation written
        return {"bytes": 2 * n * BYTES[case["x"]] + 2 * held, "flops": 4 * n}
    if op == "ln_forward":
        moved = n * (BYTES[case["x"]] + BYTES[case["y"]]) + 2 * cols * BYTES[case["params"]] + 8 * rows
        if case["save"]:  # the checkpoint written, read and restored as bf16
            moved += 2 * held + 2 * n
        return {"bytes": moved, "flops": 8 * n}
    moved = (held if case["from8"] else n * BYTES[case["x"]]) + n * (BYTES[case["dy"]] + BYTES[case["x"]])
    return {"bytes": moved + cols * BYTES[case["params"]] + 8 * rows + 8 * cols, "flops": 15 * n}


# ----------------------------------------------------- the definition in 64 bits

def _held(x):
    """What the checkpoint of the float64 matrix x stands for."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    full = cols // BLOCK * BLOCK
    for lo, hi, width in ((0, full, BLOCK), (full, cols, cols - full)):
        if hi == lo:
            continue
        v = x[:, lo:hi].reshape(rows, -1, width)
        top = v.abs().amax(2, keepdim=True)
        e = torch.ceil(torch.log2(top / 127)).clamp(-126, 122)
        e = torch.where(127 * torch.exp2(e) < top, e + 1, e)          # log2 rounded down
        e = torch.where((127 * torch.exp2(e - 1) >= top) & (e > -126), e - 1, e)  # or up
        out[:, lo:hi] = (torch.round(v / torch.exp2(e)) * torch.exp2(e)).reshape(rows, hi - lo)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "weight_grad":
        scale = np.exp2(np.arange(256, dtype=np.float64) - 127)
        scale[255] = np.nan
        table = torch.from_numpy(scale).cuda()
        column = torch.arange(case["k"], device="cuda") // BLOCK
        x = s["q8"].double() * table[s["e8"].long()][:, column]
        w = torch.einsum("tk,tn->kn" if case["layout"] == "KxN" else "tk,tn->nk", x, s["grad"].double())
        return {"dw": w if s["old"] is None else w + s["old"].double()}
    if op == "checkpoint":
        return {"x": _held(s["inp"].double())}
    gamma, beta = s["gamma"].double(), s["beta"].double()
    if op == "ln_forward":
        x = s["inp"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPS) ** -0.5
        y = (x - mean[:, None]) * rstd[:, None] * gamma + beta
        r = {"y": y, "mean": mean, "rstd": rstd}
        if case["save"]:
            r["saved"] = _held(y.to(s["out"].dtype).double())
        return r
    if s["inp"] is not None:
        x = s["inp"].double()
    else:
        table = torch.exp2(torch.arange(256, device="cuda", dtype=torch.float64) - 127)
        x = s["q8"].double() * table[s["e8"].long()][:, torch.arange(case["cols"], device="cuda") // BLOCK]
    dy, rstd = s["grad"].double(), s["rstd"].double()[:, None]
    xhat = (x - s["mean"].double()[:, None]) * rstd
    # dx_j = rstd * sum_k (delta_jk - 1/n - xhat_j xhat_k / n) dy_k gamma_k
    g = dy * gamma
    along = torch.einsum("rc,rc->r", g, xhat)[:, None] / case["cols"]
    dx = (g - g.sum(1, keepdim=True) / case["cols"] - along * xhat) * rstd
    return {"dx": dx, "dgamma": torch.einsum("rc,rc->c", dy, xhat), "dbeta": dy.sum(0)}
