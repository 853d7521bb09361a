"""Accuracy of the layer norm operators where float32 sums can lose it, against
64 bits, with bounds relative to what the definition's own operands hold: a row's
deviations from its mean, not its values."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import layer as L
from tests import layer_ref as R
from tests.layer_ref import U, U_OUT
from tests.test_gpu_layer import TYPES, Mat, _lib, as_kind, done, vec, within  # noqa: F401

pytestmark = pytest.mark.gpu

# widths of every kernel: narrow, aligned and not, groups of eight shifted,
# wider than the rings take; few are powers of two, whose 1/n is exact
WIDTHS = [40, 96, 100, 777, 1536, 2049, 3333, 4096, 5120, 8200, 12288, 16400]
PLACES = [(0, 0), (3, 1)]                           # pitch beyond the width, first element


def levels(rng, rows, cols, spread):
    """Rows about a level of full mantissa between 1000 and 2000."""
    level = rng.uniform(1000, 2000, size=(rows, 1)).astype(np.float32)
    return (level + spread * rng.normal(size=(rows, cols))).astype(np.float32)


def forward(x, xt, yt, gamma, beta, eps, pad, off):
    rows, cols = x.shape
    X, Y = Mat(rows, cols, xt, pad, off, x), Mat(rows, cols, yt, pad, off)
    mean, rstd = Mat(1, rows, "f32"), Mat(1, rows, "f32")
    done(L.gemm_layernorm_forward(rows, cols, X.ptr, X.ld, TYPES[xt], vec(gamma, "f32"), vec(beta, "f32"),
                                  TYPES["f32"], eps, Y.ptr, Y.ld, TYPES[yt], mean.ptr, rstd.ptr))
    return Y.host(), mean.host()[0], rstd.host()[0]


def forward_bounds(x, gamma, beta, eps, y_type):
    """(y, mean, rstd) error bounds.  A first mean is off by the roundings of its
    sum; the deviations d from it are single subtractions, and their own average
    takes that error out again, up to its roundings, which are relative to the
    deviations."""
    y, mean, rstd = R.ln_forward(x, gamma, beta, eps)
    x = x.astype(np.float64)
    depth = R._depth(x.shape[1]) + 2                # additions, 1/n and its product
    first = depth * U * np.abs(x).mean(1)           # error of the first mean
    d = np.abs(x - mean[:, None]) + first[:, None]  # magnitude of a deviation, at most
    c_err = (depth + 1) * U * d.mean(1)             # of their average: that of each d, and the additions'
    d_err = U * d + c_err[:, None] + 2 * U * (d + first[:, None])
    # the variance is the average of d^2 (each off by 3 U of itself) less the
    # average's square, which is at most (1.01 first)^2
    var_err = (depth + 5) * U * (d ** 2).mean(1) + 4 * first * c_err + 4 * U * first ** 2
    r_rel = var_err * rstd ** 2 / 2 * 1.01 + 4 * U
    y_err = np.abs(gamma) * (rstd[:, None] * d_err + np.abs(x - mean[:, None]) * rstd[:, None] * (r_rel[:, None] + 3 * U))
    y_err = y_err * 1.01 + 2 * U * (np.abs(y) + np.abs(beta))
    return y_err + (np.abs(y) + y_err) * U_OUT[y_type], c_err + U * np.abs(mean) * 1.01, rstd * r_rel


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("spread", [0.0, 0.01, 1.0])
def test_layernorm_forward_of_a_mean_far_above_the_deviations(cols, spread):
    """Rows about 1000 to 2000 with deviations of nothing, 0.01 and 1: y keeps
    the digits of the deviations, and a constant row gives beta."""
    rng = np.random.default_rng(cols)
    x = levels(rng, 24, cols, spread)
    gamma, beta = as_kind(1 + 0.2 * rng.normal(size=cols), "f32"), as_kind(0.2 * rng.normal(size=cols), "f32")
    for pad, off in PLACES:
        for b in (beta, np.zeros(cols, np.float32)):
            y, mean, rstd = forward(x, "f32", "f32", gamma, b, 1e-5, pad, off)
            want, m, s = R.ln_forward(x, gamma, b, 1e-5)
            by, bm, bs = forward_bounds(x, gamma, b, 1e-5, "f32")
            within(mean, m, bm)
            within(rstd, s, bs)
            within(y, want, by)


def backward_bounds(x, mean, rstd, gamma, dy, dx_type):
    """(dx, dgamma, dbeta) error bounds with xh two roundings of x - mean and its
    product with rstd (each relative to xh), and the sums over the rows at most
    a chain of all of them."""
    dx, _, _ = R.ln_backward(x, mean, rstd, gamma, dy)
    x, dy, m, s = (a.astype(np.float64) for a in (x, dy, mean, rstd))
    rows, depth = x.shape[0], R._depth(x.shape[1])
    s = s[:, None]
    xh = np.abs((x - m[:, None]) * s)
    xh_err = 2.01 * U * xh
    g = np.abs(dy * gamma)
    b = (g * xh).mean(1, keepdims=True)
    a_err = (depth + 4) * U * g.mean(1, keepdims=True)
    b_err = (depth + 6) * U * b + (g * xh_err).mean(1, keepdims=True)
    err = s * (6 * U * (g + g.mean(1, keepdims=True) + xh * b) + a_err + xh * b_err + xh_err * b)
    err = err + (np.abs(dx) + err) * U_OUT[dx_type]
    return (err, (np.abs(dy) * ((rows + 1) * U * xh + xh_err)).sum(0) * 1.01,
            (rows + 1) * U * np.abs(dy).sum(0) * 1.01)


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("xt,gt,ot", [("f32", "bf16", "f32"), ("f32", "f32", "f32"), ("bf16", "bf16", "bf16"),
                                      ("q8", "bf16", "f32")])
def test_layernorm_backward_of_a_mean_far_above_the_deviations(cols, xt, gt, ot):
    """xh has the digits of x - mean, not those of mean: dgamma of one row is
    dy * xh, of a few rows their sum."""
    rng = np.random.default_rng(cols + 1)
    for rows in (1, 3, 40):
        for pad, off in PLACES:
            X = Q = E = None
            if xt == "q8":
                q = rng.integers(90, 128, size=(rows, cols)).astype(np.int8)
                e = np.full((rows, -(-cols // 32)), 127, np.uint8)
                x = R.q8_values(q, e)
                Q, E = Mat(rows, cols, "s8", pad, off, q), Mat(rows, e.shape[1], "u8", pad, off, e)
            else:
                x = levels(rng, rows, cols, 1.0) if xt == "f32" else as_kind(100 + rng.normal(size=(rows, cols)), xt)
                X = Mat(rows, cols, xt, pad, off, x)
            gamma = as_kind(1 + 0.2 * rng.normal(size=cols), "f32")
            _, m, s = R.ln_forward(x, gamma, 0, 1e-5)
            # the statistics with full mantissas, as a forward pass gives them
            m, s = (m * (1 + 2.0 ** -20 * rng.uniform(size=rows))).astype(np.float32), s.astype(np.float32)
            dy = as_kind(rng.normal(size=(rows, cols)), gt)
            D, O = Mat(rows, cols, gt, pad, off, dy), Mat(rows, cols, ot, pad, off)
            dg, db = Mat(1, cols, "f32"), Mat(1, cols, "f32")
            done(L.gemm_layernorm_backward(
                rows, cols, X.ptr if X else None, X.ld if X else 0, TYPES[ot], Q.ptr if Q else None, Q.ld if Q else 0,
                E.ptr if E else None, E.ld if E else 0, vec(gamma, "f32"), TYPES["f32"], vec(m, "f32"), vec(s, "f32"),
                D.ptr, D.ld, TYPES[gt], O.ptr, O.ld, TYPES[ot], dg.ptr, db.ptr))
            want = R.ln_backward(x, m, s, gamma, dy)
            bound = backward_bounds(x, m, s, gamma, dy, ot)
            within(dg.host()[0], want[1], bound[1])
            within(db.host()[0], want[2], bound[2])
            within(O.host(), want[0], bound[0])


@pytest.mark.parametrize("rows,cols", [(5000, 96), (4000, 777), (3000, 1536), (2000, 5120), (1500, 5121), (700, 12288)])
def test_layernorm_forward_of_rows_of_both_kinds(rows, cols):
    """Blocks walk many rows, some with a mean far above their deviations, in
    no order: each keeps its own digits, and its own statistics."""
    rng = np.random.default_rng(rows)
    x = rng.normal(size=(rows, cols)).astype(np.float32)
    far = rng.random(rows) < 0.4
    x[far] = levels(rng, int(far.sum()), cols, 0.5)
    x[rng.integers(0, rows, size=20)] = 1234.567
    gamma, beta = as_kind(1 + 0.2 * rng.normal(size=cols), "f32"), as_kind(0.2 * rng.normal(size=cols), "f32")
    y, mean, rstd = forward(x, "f32", "f32", gamma, beta, 1e-5, 0, 0)
    want, m, s = R.ln_forward(x, gamma, beta, 1e-5)
    by, bm, bs = forward_bounds(x, gamma, beta, 1e-5, "f32")
    within(mean, m, bm)
    within(rstd, s, bs)
    within(y, want, by)
