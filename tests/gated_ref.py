"""The gated feed-forward block's gate and dropout in 64 bits (numpy, no CUDA),
and the error bounds of their float32 computation, for the tests.

Bounds.  A float32 sum of bf16 products is off by at most 2^-20 of the
products' magnitudes' sum (the GEMMs' contract).  The activations' float32
forms are off by at most 2^-18 |g|, their slopes by at most 2^-18: an
exponential of x is off by (2 + 1.2 |x|) 2^-23 of itself and enters the
logistic function s times s (1 - s), where (2 + 1.2 |x|) s (1 - s) < 0.7; a
quotient by two units, erfc by a few; the slopes' second factors x s (1 - s)
and g exp(-g^2 / 2) stay below 0.7, and their relative errors times themselves
below 2^-19.  No slope is above 1.13."""
import numpy as np
from scipy import special

from tests import layer_ref as R

SUM = 2.0 ** -20
ACT = 2.0 ** -18
TOP_SLOPE = 1.13
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]


def act(g, kind):
    """(act(g), act'(g)) in 64 bits."""
    g = np.asarray(g, np.float64)
    if kind == "relu":
        return np.maximum(g, 0), (g > 0).astype(np.float64)
    if kind == "silu":
        s = special.expit(g)
        return g * s, s * (1 + g * special.expit(-g))
    if kind == "gelu":
        p = special.ndtr(g)
        return g * p, p + g * np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
    z = np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3)
    dz = np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * g ** 2)
    s, t = special.expit(2 * z), special.expit(-2 * z)
    return g * s, s + g * 2 * s * t * dz


def _bf16(err, ref):
    return err + (np.abs(ref) + err) * R.U_OUT["bf16"] + 2.0 ** -133


def product(a, b):
    """a . b in 64 bits and the bound of its float32 sum."""
    a, b = a.astype(np.float64), b.astype(np.float64)
    return a @ b, SUM * (np.abs(a) @ np.abs(b))


def forward(x, wg, wu, kind):
    """[(H, bound), (G, bound), (U, bound)] of x (T x K) and K x F weights."""
    g, eg = product(x, wg)
    u, eu = product(x, wu)
    a, _ = act(g, kind)
    err = TOP_SLOPE * eg * (np.abs(u) + eu) + np.abs(a) * eu + ACT * np.abs(g * u) + 2.0 ** -22 * np.abs(a * u)
    return [(a * u, _bf16(err, a * u)), (g, _bf16(eg, g)), (u, _bf16(eu, u))]


def backward(dh, edh, g, u, kind):
    """[(dG, bound), (dU, bound), (act(G) U, bound in float32)]; edh: dh's own error."""
    dh, g, u = (np.asarray(v, np.float64) for v in (dh, g, u))
    a, s = act(g, kind)
    dg, du = dh * u * s, dh * a
    eg = (np.abs(dh) + edh) * np.abs(u) * ACT + edh * np.abs(u * s) + 2.0 ** -22 * np.abs(dg)
    eu = (np.abs(dh) + edh) * np.abs(g) * ACT + edh * np.abs(a) + 2.0 ** -22 * np.abs(du)
    return [(dg, _bf16(eg, dg)), (du, _bf16(eu, du)), (a * u, ACT * np.abs(g * u) + 2.0 ** -22 * np.abs(a * u))]


def held_ok(q, e, h, err):
    """Whether (q, e) is the checkpoint of a matrix within err of h: the least
    exponent of such values, every byte within half a step and that error."""
    rows, cols = h.shape
    blocks = -(-cols // R.BLOCK)

    def tops(v):
        return np.pad(v, ((0, 0), (0, blocks * R.BLOCK - cols))).reshape(rows, blocks, -1).max(2)

    def exponent(top):
        m, x = np.frexp(top)
        return np.where(top == 0, -126, np.clip(np.where(m > 127 / 128, x - 6, x - 7), -126, 122))
    lo, hi = exponent(np.maximum(tops(np.abs(h) - err), 0)), exponent(tops(np.abs(h) + err))
    E = e.astype(np.int64) - 127
    if not ((E >= lo) & (E <= hi)).all():
        return False
    step = np.repeat(np.exp2(E.astype(np.float64)), R.BLOCK, axis=1)[:, :cols]
    return (np.abs(q * step - h) <= step / 2 + err).all()


# --------------------------------------------------------------------- dropout

def philox(c, k):
    """Philox4x32-10 of counters c (4 x n, uint64 below 2^32) and key k."""
    c = [np.asarray(v, np.uint64) for v in c]
    low, up = np.uint64(0xFFFFFFFF), np.uint64(32)
    for r in range(10):
        k0, k1 = (np.uint64((int(k[i]) + r * w) % 2 ** 32) for i, w in enumerate((0x9E3779B9, 0xBB67AE85)))
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> up) ^ c[1] ^ k0, b & low, (a >> up) ^ c[3] ^ k1, a & low]
    return np.stack(c)


def threshold(p):
    return int(np.rint(np.float64(np.float32(p)) * 65536))


def keep(rows, cols, p, seed, step):
    """Which values dropout keeps."""
    groups = -(-cols // 8)
    r, g = np.meshgrid(np.arange(rows, dtype=np.uint64), np.arange(groups, dtype=np.uint64), indexing="ij")
    step %= 2 ** 64
    w = philox([g.ravel(), r.ravel(), np.full(r.size, step % 2 ** 32), np.full(r.size, step >> 32)],
               (seed % 2 ** 32, seed >> 32))
    n = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 1)          # word, half, group
    return n.transpose(2, 0, 1).reshape(rows, -1)[:, :cols] >= threshold(p)


def dropout(x, residual, p, seed, step, y_type):
    """(y, bound): a product, a sum and their roundings in float32, then the type's."""
    x = x.astype(np.float64)
    t = threshold(p)
    v = np.where(keep(*x.shape, p, seed, step), x * (65536 / max(65536 - t, 1)), 0)
    b = 0 if residual is None else residual.astype(np.float64)
    y = v + b
    err = 3 * R.U * (np.abs(v) + np.abs(b)) + 2.0 ** -149
    return y, err + (np.abs(y) + err) * R.U_OUT[y_type] + (2.0 ** -133 if y_type == "bf16" else 0)
