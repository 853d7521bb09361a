"""The operators of a gated feed-forward block, as measured cases.

The second half of a transformer layer computes, of the normalised tokens X,

    G = X . Wg,  U = X . Wu,  H = act(G) * U,  O = H . Wd,
    y = x + dropout(O),

and goes back through the same.  Beside the GEMMs, the layer norm and the
weight gradients, which the library has, that takes:

  gated_forward        H in one kernel, from one token (serving) to a full
                       micro-batch; G and U kept in bf16 if a backward pass
                       follows;
  gated_backward       dG = dH * U * act'(G) and dU = dH * act(G), and the
                       8-bit checkpoint of act(G) * U, from which Wd's gradient
                       is taken;
  gated_down_backward  the same with dH = dO . Wd^T taken in the same kernel;
  dropout              y = residual + keep * x / (1 - p), and its gradient;
                       keep is a function of (seed, step, row, column).

The checkpoint holds blocks of 32 consecutive values of a row: a power of two
2^E, E the least exponent >= -126 with max|x| <= 127 * 2^E, and 32 signed
bytes round_half_even(x / 2^E).

Dropout's generator is Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel
random numbers: as easy as 1, 2, 3", 2011) with key seed and counter
(column / 8, row, step): its 128 bits are the 16-bit numbers of eight
neighbouring values, the lowest bits the first one's.  A value is kept where
its number is at least round(65536 p).

``own`` selects between the plain form (elementary torch operations in 32
bits) and the library's calls.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]
LARGEST_MACS = 8192 * 4096 * 11008
LARGEST_ELEMENTS = 8192 * 12288


def listed():
    return [
        # one token being generated: the weights' bytes and the call's latency
        {"name": "gated fwd 1t 4096x11008", "op": "gated_forward", "tokens": 1, "k": 4096, "f": 11008,
         "layout": "NxK", "act": "silu", "save": False, "joined": False, "pad": 0},
        # a batch of sequences, a token each: the weights' bytes
        {"name": "gated fwd 48t 4096x11008", "op": "gated_forward", "tokens": 48, "k": 4096, "f": 11008,
         "layout": "KxN", "act": "gelu_tanh", "save": False, "joined": True, "pad": 0},
        # a short prompt through a layer of odd widths: no row 16-byte aligned
        {"name": "gated fwd 300t 777x1501", "op": "gated_forward", "tokens": 300, "k": 777, "f": 1501,
         "layout": "KxN", "act": "gelu", "save": True, "joined": True, "pad": 0},
        # a short training micro-batch
        {"name": "gated fwd 2048t 4096x11008 saved", "op": "gated_forward", "tokens": 2048, "k": 4096, "f": 11008,
         "layout": "KxN", "act": "silu", "save": True, "joined": True, "pad": 0},
        # a full training micro-batch: the tensor cores
        {"name": "gated fwd 8192t 4096x11008 saved", "op": "gated_forward", "tokens": 8192, "k": 4096, "f": 11008,
         "layout": "KxN", "act": "silu", "save": True, "joined": True, "pad": 0},
        # the gate's gradient where dH comes from elsewhere (summed over devices, say), odd width
        {"name": "gated bwd 1000x1501", "op": "gated_backward", "tokens": 1000, "f": 1501, "act": "gelu",
         "held": True, "joined": True, "pad": 0},
        # the same over a full micro-batch: memory-bound
        {"name": "gated bwd 8192x11008", "op": "gated_backward", "tokens": 8192, "f": 11008, "act": "silu",
         "held": True, "joined": True, "pad": 0},
        # the down projection's product and the gate's gradient, odd widths
        {"name": "gated down bwd 1000t 777x1501", "op": "gated_down_backward", "tokens": 1000, "n": 777, "f": 1501,
         "layout": "KxN", "act": "gelu_tanh", "held": True, "joined": True, "pad": 0},
        # ... of a full micro-batch: the tensor cores, and 9 bytes an element of H beside them
        {"name": "gated down bwd 8192t 4096x11008", "op": "gated_down_backward", "tokens": 8192, "n": 4096, "f": 11008,
         "layout": "KxN", "act": "silu", "held": True, "joined": True, "pad": 0},
        # a small batch: latency
        {"name": "dropout 16x4096", "op": "dropout", "rows": 16, "cols": 4096, "x": "bf16", "y": "bf16", "p": 0.1,
         "back": False, "residual": True, "pad": 0},
        # a block's output into a float32 residual stream over a full micro-batch: memory-bound
        {"name": "dropout 8192x12288 into f32", "op": "dropout", "rows": 8192, "cols": 12288, "x": "bf16", "y": "f32",
         "p": 0.1, "back": False, "residual": True, "pad": 0},
        # the gradient of a float32 residual stream of odd width, going back
        {"name": "dropout back 2560x777", "op": "dropout", "rows": 2560, "cols": 777, "x": "bf16", "y": "f32",
         "p": 0.25, "back": True, "residual": False, "pad": 0},
    ]


def _size(rng, lo, hi, step=8):
    """A size between lo and hi, spread over its logarithm; two in three a multiple of `step`, else any."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 2 / 3 and v > step:
        v = v // step * step
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["gated_forward", "gated_forward", "gated_backward", "gated_down_backward", "dropout"])
    pad = rng.choice([0, 0, 0, 8, 32, 5])
    if op == "dropout":
        while True:
            rows, cols = _size(rng, 1, 16384), _size(rng, 64, 12288)
            if rows * cols <= LARGEST_ELEMENTS:
                break
        back = rng.random() < 0.4
        return {"op": op, "rows": rows, "cols": cols, "x": rng.choice(["bf16", "f32"]), "y": rng.choice(["bf16", "f32"]),
                "p": rng.choice([0.0, 0.05, 0.1, 0.3, 0.5]), "back": back, "residual": not back and rng.random() < 0.8,
                "pad": pad}
    case = {"op": op, "act": rng.choice(ACTS), "joined": rng.random() < 0.6, "pad": pad}
    if op == "gated_backward":
        while True:
            t, f = _size(rng, 1, 16384), _size(rng, 64, 12288)
            if t * f <= LARGEST_ELEMENTS:
                break
        case.update(tokens=t, f=f, held=rng.random() < 0.7)
        return case
    while True:
        t, k, f = _size(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 12288)
        if t * k * f <= LARGEST_MACS:
            break
    case.update(tokens=t, f=f, layout=rng.choice(["KxN", "NxK"]))
    if op == "gated_forward":
        case.update(k=k, save=rng.random() < 0.5)
    else:
        case.update(n=k, held=rng.random() < 0.7)
    return case


# ------------------------------------------------------------------- inputs

def _rows(rows, cols, pad, dtype, fill=None):
    """A rows x cols matrix that is the left part of a buffer `pad` columns wider."""
    buf = torch.zeros((rows, cols + pad), dtype=dtype, device="cuda")
    if fill is not None:
        buf[:, :cols].copy_(fill)
    return buf[:, :cols]


def _two(rows, cols, case, dtype=torch.bfloat16):
    """Two rows x cols matrices: the halves of one (joined), or apart."""
    if case["joined"]:
        both = _rows(rows, 2 * cols, case["pad"], dtype)
        return both[:, :cols], both[:, cols:]
    return _rows(rows, cols, case["pad"], dtype), _rows(rows, cols, case["pad"], dtype)


def _gradients(gen, rows, cols):
    """Gradients of small magnitude; one row in sixteen is a masked token's, all zero."""
    r = dict(generator=gen, device="cuda", dtype=torch.float32)
    g = 1e-3 * torch.randn((rows, cols), **r)
    return torch.where(torch.rand((rows, 1), **r) < 1 / 16, torch.zeros_like(g), g)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 6151 + 29)
    r = dict(generator=gen, device="cuda", dtype=torch.float32)
    s = dict(case)
    op, pad, bf = case["op"], case["pad"], torch.bfloat16
    if op == "dropout":
        rows, cols = case["rows"], case["cols"]
        xt, yt = DTYPES[case["x"]], DTYPES[case["y"]]
        s["seed"], s["step"] = int(seed) * 0x9E3779B97F4A7C15 % 2 ** 64, int(seed) % 1000 + 2 ** 33
        if case["back"]:
            s["inp"] = _rows(rows, cols, pad, yt, _gradients(gen, rows, cols))
            s["res"], s["out"] = None, _rows(rows, cols, pad, xt)
        else:
            s["inp"] = _rows(rows, cols, pad, xt, torch.randn((rows, cols), **r))
            s["res"] = _rows(rows, cols, pad, yt, 2 * torch.randn((rows, cols), **r)) if case["residual"] else None
            s["out"] = _rows(rows, cols, pad, yt)
        return s
    t, f = case["tokens"], case["f"]
    if op == "gated_forward":
        k, kn = case["k"], case["layout"] == "KxN"
        # normalised tokens: unit variance, channels of different gain, one in a hundred an outlier
        gain = torch.exp(0.3 * torch.randn(k, **r))
        gain = torch.where(torch.rand(k, **r) < 0.01, gain * 8, gain)
        s["inp"] = _rows(t, k, pad, bf, torch.randn((t, k), **r) * gain)
        shape = (k, f) if kn else (f, k)
        if case["joined"]:  # gate and up projection side by side in one matrix
            w = _rows(k, 2 * f, pad, bf) if kn else _rows(2 * f, k, pad, bf)
            s["wg"], s["wu"] = (w[:, :f], w[:, f:]) if kn else (w[:f], w[f:])
        else:
            s["wg"], s["wu"] = _rows(*shape, pad, bf), _rows(*shape, pad, bf)
        for w in (s["wg"], s["wu"]):
            w.copy_(torch.randn(shape, **r) / k ** 0.5)
        s["h"] = _rows(t, f, pad, bf)
        s["g"], s["u"] = _two(t, f, case) if case["save"] else (None, None)
        return s
    s["g"], s["u"] = _two(t, f, case)
    s["g"].copy_(1.2 * torch.randn((t, f), **r))
    s["u"].copy_(1.2 * torch.randn((t, f), **r))
    s["dg"], s["du"] = _two(t, f, case)
    s["q8"] = s["e8"] = s["restored"] = None
    if case["held"]:
        s["q8"] = torch.zeros((t, f), dtype=torch.int8, device="cuda")
        s["e8"] = torch.zeros((t, -(-f // BLOCK)), dtype=torch.uint8, device="cuda")
        s["restored"] = torch.zeros((t, f), dtype=bf, device="cuda")
    if op == "gated_backward":
        s["grad"] = _rows(t, f, pad, bf, _gradients(gen, t, f))
        return s
    n = case["n"]
    s["grad"] = _rows(t, n, pad, bf, _gradients(gen, t, n))
    shape = (f, n) if case["layout"] == "KxN" else (n, f)
    s["wd"] = _rows(*shape, pad, bf, torch.randn(shape, **r) / n ** 0.5)
    return s


# ---------------------------------------------------------------- plain form

def _activation(g, act):
    """(act(g), act'(g)) of the float32 matrix g."""
    if act == "relu":
        on = g > 0
        return torch.where(on, g, torch.zeros_like(g)), on.float()
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        return g * sig, sig * (1 + g * (1 - sig))
    if act == "gelu":
        phi = 0.5 * torch.erfc(-g * math.sqrt(0.5))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    c = math.sqrt(2 / math.pi)
    # 0.5 * (1 + tanh(z)) = 1 / (1 + exp(-2 z))
    sig = 1 / (1 + torch.exp(-2 * c * (g + 0.044715 * g * g * g)))
    return g * sig, sig + g * sig * (1 - sig) * 2 * c * (1 + 3 * 0.044715 * g * g)


def _held(x):
    """What the checkpoint of the float32 matrix x stands for, in bf16."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    v = torch.nn.functional.pad(x, (0, blocks * BLOCK - cols)).view(rows, blocks, BLOCK)
    top = v.abs().amax(2, keepdim=True)
    m, ex = torch.frexp(top)                          # top = m * 2^ex, 0.5 <= m < 1
    e = torch.where(m > 127 / 128, ex - 6, ex - 7).clamp(-126, 122).to(torch.int32)
    back, there = ((e + 127) << 23).view(torch.float32), ((127 - e) << 23).view(torch.float32)
    return (torch.round(v * there) * back).view(rows, -1)[:, :cols].to(torch.bfloat16)


def _keep(rows, cols, p, seed, step):
    """Which values dropout keeps."""
    r = dict(device="cuda", dtype=torch.int64)
    low = 0xFFFFFFFF
    groups = -(-cols // 8)
    c0 = torch.arange(groups, **r)[None, :].expand(rows, groups)
    c1 = torch.arange(rows, **r)[:, None].expand(rows, groups)
    c2, c3 = torch.full_like(c0, step & low), torch.full_like(c0, step >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 2)
    numbers = torch.stack([words & 0xFFFF, words >> 16], 3).view(rows, -1)[:, :cols]
    return numbers >= _threshold(p)


def _threshold(p):
    return round(float(np.float32(p)) * 65536)


def _plain(s):
    op = s["op"]
    if op == "dropout":
        x = s["inp"].float()
        keep = _keep(s["rows"], s["cols"], s["p"], s["seed"], s["step"])
        v = torch.where(keep, x * (65536 / (65536 - _threshold(s["p"]))), torch.zeros_like(x))
        if s["res"] is not None:
            v = s["res"].float() + v
        return {"dx" if s["back"] else "y": v.to(s["out"].dtype)}
    bf = torch.bfloat16
    if op == "gated_forward":
        x, wg, wu = s["inp"].float(), s["wg"].float(), s["wu"].float()
        if s["layout"] == "NxK":
            wg, wu = wg.t(), wu.t()
        g, u = x @ wg, x @ wu
        r = {"h": (_activation(g, s["act"])[0] * u).to(bf)}
        if s["save"]:
            r.update(g=g.to(bf), u=u.to(bf))
        return r
    if op == "gated_backward":
        dh = s["grad"].float()
    else:
        wd = s["wd"].float()
        dh = s["grad"].float() @ (wd.t() if s["layout"] == "KxN" else wd)
    g, u = s["g"].float(), s["u"].float()
    a, slope = _activation(g, s["act"])
    r = {"dg": (dh * u * slope).to(bf), "du": (dh * a).to(bf)}
    if s["held"]:
        r["h"] = _held(a * u)
    return r


# ------------------------------------------------------------- library's calls

def _ours(s):
    from paper_2512_13282_gb300 import layer as L
    op = s["op"]
    if op == "dropout":
        ty = {torch.float32: L.GEMM_TYPE_F32, torch.bfloat16: L.GEMM_TYPE_BF16}
        rows, cols, x, y, res = s["rows"], s["cols"], s["inp"], s["out"], s["res"]
        if s["back"]:
            L.check(L.gemm_dropout_backward(rows, cols, x, x.stride(0), ty[x.dtype], y, y.stride(0), ty[y.dtype],
                                            s["p"], s["seed"], s["step"]))
            return {"dx": y}
        L.check(L.gemm_dropout_forward(rows, cols, x, x.stride(0), ty[x.dtype], res, res.stride(0) if res is not None
                                       else 0, y, y.stride(0), ty[y.dtype], s["p"], s["seed"], s["step"]))
        return {"y": y}
    act = {"silu": L.GEMM_ACT_SILU, "gelu": L.GEMM_ACT_GELU, "gelu_tanh": L.GEMM_ACT_GELU_TANH,
           "relu": L.GEMM_ACT_RELU}[s["act"]]
    t, f, g, u = s["tokens"], s["f"], s["g"], s["u"]
    if op != "gated_backward":
        layout = L.GEMM_B_ROW_MAJOR_KxN if s["layout"] == "KxN" else L.GEMM_B_COL_MAJOR_NxK
    if op == "gated_forward":
        x, wg, wu, h, save = s["inp"], s["wg"], s["wu"], s["h"], s["save"]
        L.check(L.gemm_gated_forward(t, s["k"], f, x, x.stride(0), wg, wg.stride(0), wu, wu.stride(0), layout, act,
                                     h, h.stride(0), g, g.stride(0) if save else 0, u, u.stride(0) if save else 0))
        return {"h": h, "g": g, "u": u} if save else {"h": h}
    dg, du, grad, q, e = s["dg"], s["du"], s["grad"], s["q8"], s["e8"]
    held = s["held"]
    rest = (g, g.stride(0), u, u.stride(0), act, dg, dg.stride(0), du, du.stride(0), q, q.stride(0) if held else 0,
            e, e.stride(0) if held else 0)
    if op == "gated_backward":
        L.check(L.gemm_gated_backward(t, f, grad, grad.stride(0), *rest))
    else:
        wd = s["wd"]
        L.check(L.gemm_gated_down_backward(t, s["n"], f, grad, grad.stride(0), wd, wd.stride(0), layout, *rest))
    r = {"dg": dg, "du": du}
    if held:
        back = s["restored"]
        L.check(L.gemm_q8_restore(t, f, q, q.stride(0), e, e.stride(0), back, back.stride(0), L.GEMM_TYPE_BF16))
        r["h"] = back
    return r


def run(state):
    return _ours(state) if own else _plain(state)


# ------------------------------------------------------------------ cost

def work(case):
    op = case["op"]
    if op == "dropout":
        n = case["rows"] * case["cols"]
        moved = BYTES[case["x"]] + BYTES[case["y"]] * (2 if case["residual"] else 1)
        return {"bytes": n * moved, "flops": 2 * n}
    t, f = case["tokens"], case["f"]
    if op == "gated_forward":
        k = case["k"]
        return {"bytes": 2 * (t * k + 2 * k * f + t * f * (3 if case["save"] else 1)), "flops": 4 * t * k * f}
    moved = 8 * t * f  # G and U read, dG and dU written
    if case["held"]:   # the checkpoint written, read and restored as bf16
        moved += 2 * t * (f + -(-f // BLOCK)) + 2 * t * f
    if op == "gated_backward":
        return {"bytes": moved + 2 * t * f, "flops": 20 * t * f}
    n = case["n"]
    return {"bytes": moved + 2 * (t * n + n * f), "flops": 2 * t * n * f}


# ----------------------------------------------------- the definition in 64 bits

def _act64(g, act):
    if act == "relu":
        return g.clamp(min=0), torch.heaviside(g, torch.zeros((), dtype=g.dtype, device=g.device))
    if act == "silu":
        s = torch.special.expit(g)
        return s * g, s + s * (1 - s) * g
    if act == "gelu":
        n = torch.special.ndtr(g)
        return n * g, n + g * torch.exp(-g ** 2 / 2) / (2 * torch.pi) ** 0.5
    z = (2 / torch.pi) ** 0.5 * (g + 0.044715 * g ** 3)
    dz = (2 / torch.pi) ** 0.5 * (1 + 0.134145 * g ** 2)
    th = torch.tanh(z)
    return g * (1 + th) / 2, (1 + th) / 2 + g / 2 / torch.cosh(z) ** 2 * dz


def _kept64(rows, cols, p, seed, step):
    """The same generator on the host, in unsigned 64-bit arithmetic."""
    groups, low, up = -(-cols // 8), np.uint64(0xFFFFFFFF), np.uint64(32)
    x = np.tile(np.arange(groups, dtype=np.uint64), rows)
    y = np.repeat(np.arange(rows, dtype=np.uint64), groups)
    z, w = np.full_like(x, step % 2 ** 32), np.full_like(x, step // 2 ** 32)
    for i in range(10):
        key = [np.uint64((seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32), np.uint64((seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32)]
        m, n = x * np.uint64(0xD2511F53), z * np.uint64(0xCD9E8D57)
        x, y, z, w = (n >> up) ^ y ^ key[0], n & low, (m >> up) ^ w ^ key[1], m & low
    bits = np.stack([x, y, z, w], 1).astype("<u4").view("<u2").reshape(rows, -1)[:, :cols]
    return torch.from_numpy(bits.astype(np.int32) >= int(np.rint(np.float64(np.float32(p)) * 65536))).cuda()


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "dropout":
        kept = _kept64(case["rows"], case["cols"], case["p"], s["seed"], s["step"]).double()
        share = 1 - np.rint(np.float64(np.float32(case["p"])) * 65536) / 65536
        v = s["inp"].double() * kept / share
        if s["res"] is not None:
            v += s["res"].double()
        return {"dx" if case["back"] else "y": v}
    if op == "gated_forward":
        to = "tk,kf->tf" if case["layout"] == "KxN" else "tk,fk->tf"
        x = s["inp"].double()
        g, u = (torch.einsum(to, x, s[w].double()) for w in ("wg", "wu"))
        r = {"h": u * _act64(g, case["act"])[0]}
        if case["save"]:
            r.update(g=g, u=u)
        return r
    if op == "gated_backward":
        dh = s["grad"].double()
    else:
        dh = torch.einsum("tn,fn->tf" if case["layout"] == "KxN" else "tn,nf->tf", s["grad"].double(), s["wd"].double())
    g, u = s["g"].double(), s["u"].double()
    a, slope = _act64(g, case["act"])
    r = {"dg": slope * u * dh, "du": a * dh}
    if case["held"]:
        r["h"] = None  # a value next to a step's border goes by the last bit of its float32 form
    return r
