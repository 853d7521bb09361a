"""Sums of the layer operators that must come out exactly, and matrices whose
rows lie more than 2^31 elements apart."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import layer as L
from tests import layer_ref as R
from tests.test_gpu_layer import EPS, TYPES, Mat, _lib, as_kind, done, vec, within  # noqa: F401
from tests.test_gpu_layer_accuracy import backward_bounds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [
    (3, 4096), (4, 777), (5, 777), (40, 16400), (300, 20000), (310, 16384), (600, 12288), (700, 40), (1000, 1500),
    (1500, 8192), (2500, 128), (3000, 5120), (1300, 5690), (4900, 2304), (5000, 4096), (8000, 1024), (9000, 141),
    (20000, 100), (20000, 512)])
@pytest.mark.parametrize("xt,gt,ot", [("bf16", "bf16", "bf16"), ("f32", "f32", "f32"), ("q8", "bf16", "f32")])
def test_parameter_gradients_of_integers_are_exact(rows, cols, xt, gt, ot):
    """Mean 0, 1/std 1 and small integers in x and dy: every sum is below 2^24,
    so dgamma = sum(dy * x) and dbeta = sum(dy) are those integers whatever the
    order of the additions.  Each row adds to both, so that no row, and no
    block's partial sums, can be lost or taken twice unnoticed."""
    rng = np.random.default_rng(rows + cols)
    x = rng.integers(-4, 5, size=(rows, cols)).astype(np.float32)
    dy = rng.integers(-4, 5, size=(rows, cols)).astype(np.float32)
    assert ((x * dy) != 0).any(1).all() and (dy != 0).any(1).all() and rows * 16 < 1 << 24
    X = Q = E = None
    if xt == "q8":
        Q, E = Mat(rows, cols, "s8", fill=x.astype(np.int8)), Mat(rows, -(-cols // 32), "u8")
        E.view.fill_(127)
    else:
        X = Mat(rows, cols, xt, fill=x)
    D, O, dg, db = Mat(rows, cols, gt, fill=dy), Mat(rows, cols, ot), Mat(1, cols, "f32"), Mat(1, cols, "f32")
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    done(L.gemm_layernorm_backward(
        rows, cols, X.ptr if X else None, cols if X else 0, TYPES[ot], Q.ptr if Q else None, cols, E.ptr if E else None,
        E.ld if E else 0, None, 0, mean, rstd, D.ptr, cols, TYPES[gt], O.ptr, cols, TYPES[ot], dg.ptr, db.ptr))
    assert np.array_equal(dg.host()[0], (x.astype(np.int64) * dy.astype(np.int64)).sum(0))
    assert np.array_equal(db.host()[0], dy.astype(np.int64).sum(0))


class Far:
    """Matrices side by side in rows of 2^26 elements and more: the last of 40
    rows starts past 2^31 elements."""

    def __init__(self, kind, rows=40, skew=8):
        dt = {"f32": torch.float32, "bf16": torch.bfloat16, "s8": torch.int8, "u8": torch.uint8}[kind]
        self.ld, self.at = (1 << 26) + skew, 0
        self.buf = torch.empty(rows * self.ld, dtype=dt, device="cuda").view(rows, self.ld)

    def put(self, rows, cols, fill=None):
        view = self.buf[:rows, self.at:self.at + cols]
        self.at += 1 << 20
        view.copy_(torch.from_numpy(np.ascontiguousarray(fill))) if fill is not None else view.zero_()
        return view


@pytest.mark.parametrize("skew,cols", [(8, 4096), (3, 4097), (8, 16392)])
def test_layernorm_offsets_past_32_bits(skew, cols):
    rng = np.random.default_rng(cols)
    rows = 40
    x, dy = (as_kind(rng.normal(size=(rows, cols)), "bf16") for _ in range(2))
    far, bytes_ = Far("bf16", rows, skew), Far("s8", rows, skew)
    exps = Far("u8", rows, skew)
    X, Y = far.put(rows, cols, x), far.put(rows, cols)
    Q, E = bytes_.put(rows, cols), exps.put(rows, -(-cols // 32))
    gamma, beta = as_kind(1 + 0.2 * rng.normal(size=cols), "f32"), as_kind(0.2 * rng.normal(size=cols), "f32")
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    done(L.gemm_layernorm_forward(rows, cols, X, far.ld, 1, vec(gamma, "f32"), vec(beta, "f32"), 0, EPS, Y, far.ld, 1,
                                  mean, rstd, Q, bytes_.ld, E, exps.ld))
    y = Y.float().cpu().numpy()
    within(y, R.ln_forward(x, gamma, beta, EPS)[0], R.ln_forward_bounds(x, gamma, beta, EPS, "bf16")[0])
    q, e = R.q8_save(y)
    assert np.array_equal(Q.cpu().numpy(), q) and np.array_equal(E.cpu().numpy(), e)
    # backward from x, and from the checkpoint as if it were x's
    D, O = far.put(rows, cols, dy), far.put(rows, cols)
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    m, s = mean.cpu().numpy(), rstd.cpu().numpy()
    for src in (x, R.q8_values(q, e)):
        from_x = src is x
        done(L.gemm_layernorm_backward(
            rows, cols, X if from_x else None, far.ld, 1, None if from_x else Q, bytes_.ld, None if from_x else E,
            exps.ld, vec(gamma, "f32"), 0, mean, rstd, D, far.ld, 1, O, far.ld, 1, dg, db))
        want, bound = R.ln_backward(src, m, s, gamma, dy), backward_bounds(src, m, s, gamma, dy, "bf16")
        within(O.float().cpu().numpy(), want[0], bound[0])
        within(dg.cpu().numpy(), want[1], bound[1])
        within(db.cpu().numpy(), want[2], bound[2])


@pytest.mark.parametrize("skew", [8, 3])
@pytest.mark.parametrize("nk", [False, True])
def test_weight_grad_offsets_past_32_bits(skew, nk):
    """Tokens of X and dY, and rows of base and dW, past 2^31 elements."""
    rng = np.random.default_rng(7)
    T, K, N = (40, 40, 72) if not nk else (40, 72, 40)
    q = rng.integers(-127, 128, size=(T, K)).astype(np.int8)
    e = rng.integers(118, 122, size=(T, -(-K // 32))).astype(np.uint8)
    dy = as_kind(rng.normal(size=(T, N)), "bf16")
    shape = (N, K) if nk else (K, N)
    base = as_kind(rng.normal(size=shape), "f32")
    s8, u8, bf, f32 = (Far(k, 40, skew) for k in ("s8", "u8", "bf16", "f32"))
    Q, E, D = s8.put(T, K, q), u8.put(T, e.shape[1], e), bf.put(T, N, dy)
    B, W = f32.put(*shape, base), f32.put(*shape)
    ref, mag = R.weight_grad(R.q8_values(q, e), dy, base, nk)
    layout = L.GEMM_B_COL_MAJOR_NxK if nk else L.GEMM_B_ROW_MAJOR_KxN
    for out in (W, B):                              # apart, then in place
        done(L.gemm_q8_weight_grad(T, K, N, Q, s8.ld, E, u8.ld, D, bf.ld, B, f32.ld, out, f32.ld, layout, 0))
        within(out.cpu().numpy(), ref, R.weight_grad_bound(ref, mag, "f32"))
    # no tokens: the base itself
    done(L.gemm_q8_weight_grad(0, K, N, None, 0, None, 0, None, 0, B, f32.ld, W, f32.ld, layout, 0))
    assert torch.equal(W, B)
