"""The layer operators' definitions in 64 bits (numpy, no CUDA), and the error
bounds of their float32 computation, for the tests."""
import numpy as np

U = 2.0 ** -24          # half a unit in the last place of a float32, relative
U_OUT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
BLOCK = 32


def bf16_round(x):
    """float32 values rounded to bf16 (nearest, ties to even), as float32."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32))


def q8_save(x):
    """(q, e) of a float32 matrix, block by block, from the definition: the
    least E >= -126 with top <= 127 * 2^E, found by trying exponents upwards."""
    rows, cols = x.shape
    q = np.zeros((rows, cols), np.int8)
    e = np.zeros((rows, -(-cols // BLOCK)), np.uint8)
    for r in range(rows):
        for b in range(e.shape[1]):
            v = x[r, b * BLOCK:(b + 1) * BLOCK].astype(np.float64)
            top = np.max(np.abs(v))
            if not np.isfinite(top):
                e[r, b] = 255
                continue
            E = -126 if top == 0 else max(-126, int(np.frexp(top)[1]) - 10)
            while top > 127 * 2.0 ** E:
                E += 1
            e[r, b] = E + 127
            limit = 63 if E == 122 else 127          # 64 * 2^122 is past float32
            q[r, b * BLOCK:(b + 1) * BLOCK] = np.clip(np.rint(v / 2.0 ** E), -limit, limit).astype(np.int8)
    return q, e


def q8_values(q, e):
    scale = np.exp2(np.arange(256, dtype=np.float64) - 127)
    scale[255] = np.nan
    scale[0] = 0
    return q.astype(np.float64) * np.repeat(scale[e], BLOCK, axis=1)[:, :q.shape[1]]


def _depth(n):
    """Longest chain of float32 additions in a sum of n values: a lane's own
    values (at least 32 lanes share a row), then the tree over lanes and warps."""
    return -(-n // 32) + 16


def ln_forward(x, gamma, beta, eps):
    x = x.astype(np.float64)
    mean = x.mean(1)
    var = ((x - mean[:, None]) ** 2).mean(1)
    rstd = 1 / np.sqrt(var + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def ln_forward_bounds(x, gamma, beta, eps, y_type):
    """(y, mean, rstd) error bounds.  The mean is off by its additions'
    roundings; the variance by those of the squared differences and by the
    mean's error squared; y by both and by its own four operations."""
    y, mean, rstd = ln_forward(x, gamma, beta, eps)
    x = np.abs(x.astype(np.float64))
    d = _depth(x.shape[1])
    m_err = (d + 2) * U * x.mean(1)
    # a difference x - mean is off by its own rounding and by the mean's error
    own = U * (x + np.abs(mean)[:, None])
    diff = own + m_err[:, None]
    # variance: the additions and squares; the mean's error, which enters
    # squared (the differences from the true mean sum to zero); the
    # differences' roundings, whose products with the differences average at
    # most the product of their root mean squares (relative: twice that)
    r_rel = ((d + 8) * U + (m_err * rstd) ** 2 + 2 * np.sqrt(np.mean(own ** 2, 1)) * rstd) / 2 + 4 * U
    xh = np.abs((y - beta) / np.where(gamma == 0, 1, gamma))
    y_err = np.abs(gamma) * rstd[:, None] * diff + np.abs(gamma) * xh * (r_rel[:, None] + 4 * U) + 2 * U * np.abs(y)
    y_err = y_err + (np.abs(y) + y_err) * U_OUT[y_type]
    return y_err, m_err + U * np.abs(mean), rstd * r_rel


def ln_backward(x, mean, rstd, gamma, dy):
    x, dy, m, s = (a.astype(np.float64) for a in (x, dy, mean, rstd))
    xh = (x - m[:, None]) * s[:, None]
    g = dy * gamma
    dx = s[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def ln_backward_bounds(x, mean, rstd, gamma, dy, dx_type):
    """(dx, dgamma, dbeta) error bounds: xh carries the rounding of x - mean
    and of its product with rstd; the averages those of their additions."""
    dx, _, _ = ln_backward(x, mean, rstd, gamma, dy)
    x, dy, m, s = (a.astype(np.float64) for a in (x, dy, mean, rstd))
    n, d = x.shape[1], _depth(x.shape[1])
    m, s = m[:, None], s[:, None]
    xh = np.abs((x - m) * s)
    xh_err = U * (np.abs(x) + np.abs(m)) * s + 3 * U * xh
    g = np.abs(dy * gamma)
    a_err = (d + 4) * U * g.mean(1, keepdims=True)
    b = (g * xh).mean(1, keepdims=True)
    b_err = (d + 6) * U * b + (g * xh_err).mean(1, keepdims=True)
    t = g + g.mean(1, keepdims=True) + xh * b
    err = s * (6 * U * t + a_err + xh * b_err + xh_err * b)
    err = err + (np.abs(dx) + err) * U_OUT[dx_type]
    rows = x.shape[0]
    dg_err = (rows + 40) * U * (np.abs(dy) * xh).sum(0) + (np.abs(dy) * xh_err).sum(0)
    return err, dg_err, (rows + 40) * U * np.abs(dy).sum(0)


def weight_grad(values, dy, base, layout_nk):
    w = values.T @ dy.astype(np.float64)
    mag = np.abs(values).T @ np.abs(dy.astype(np.float64))
    if layout_nk:
        w, mag = w.T, mag.T
    if base is not None:
        w, mag = w + base.astype(np.float64), mag + np.abs(base.astype(np.float64))
    return w, mag


def weight_grad_bound(ref, mag, w_type):
    """The header's accuracy contract (float32), with the final rounding of the type."""
    err = 2.0 ** -20 * mag
    return err + (np.abs(ref) + err) * U_OUT[w_type]
