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
