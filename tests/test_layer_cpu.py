"""Host-side checks of the layer operators' C ABI that need no GPU: every
declared function is exported, bad arguments are refused before the device is
touched, and empty problems are no-ops."""
import numpy as np
import pytest

from paper_2512_13282_gb300 import build as B
from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from tests import layer_ref as R

P = 0x1000  # an aligned address that is never dereferenced: validation fails first
F32, BF16 = L.GEMM_TYPE_F32, L.GEMM_TYPE_BF16
BAD, OK = G.GEMM_ERR_INVALID_ARG, G.GEMM_OK


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return L.library()


def fwd(rows=4, cols=40, x=P, ldx=40, xt=BF16, gamma=P, beta=P, pt=F32, eps=1e-5, y=P, ldy=40, yt=BF16, mean=P,
        rstd=P, q=0, ldq=0, e=0, lde=0):
    return L.gemm_layernorm_forward(rows, cols, x, ldx, xt, gamma, beta, pt, eps, y, ldy, yt, mean, rstd, q, ldq, e,
                                    lde, stream=0)


def bwd(rows=4, cols=40, x=P, ldx=40, xt=BF16, q=0, ldq=0, e=0, lde=0, gamma=P, pt=F32, mean=P, rstd=P, dy=P, lddy=40,
        gt=BF16, dx=P, lddx=40, dt=BF16, dgamma=P, dbeta=P):
    return L.gemm_layernorm_backward(rows, cols, x, ldx, xt, q, ldq, e, lde, gamma, pt, mean, rstd, dy, lddy, gt, dx,
                                     lddx, dt, dgamma, dbeta, stream=0)


def wgrad(T=4, K=40, N=8, q=P, ldq=40, e=P, lde=2, dY=P, lddy=8, base=0, ldbase=0, dW=P, ldw=8,
          layout=L.GEMM_B_ROW_MAJOR_KxN, wt=F32):
    return L.gemm_q8_weight_grad(T, K, N, q, ldq, e, lde, dY, lddy, base, ldbase, dW, ldw, layout, wt, stream=0)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-1), dict(xt=2), dict(yt=-1), dict(pt=7), dict(eps=-1.0), dict(eps=float("nan")),
    dict(x=0), dict(y=0), dict(ldx=39), dict(ldy=39), dict(x=P + 1), dict(y=P + 2, yt=F32), dict(gamma=P + 2),
    dict(beta=P + 1, pt=BF16), dict(mean=P + 2), dict(rstd=P + 1), dict(q=P, ldq=40), dict(e=P, lde=2),
    dict(q=P, ldq=39, e=P, lde=2), dict(q=P, ldq=40, e=P, lde=1)])
def test_layernorm_forward_refusals(bad):
    assert fwd(**bad) == BAD, bad


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-1), dict(xt=F32), dict(gt=3), dict(dt=9), dict(pt=2), dict(x=0), dict(q=P, e=P),
    dict(x=0, q=P, ldq=40), dict(x=0, q=P, ldq=39, e=P, lde=2), dict(x=0, q=P, ldq=40, e=P, lde=1), dict(ldx=39),
    dict(dy=0), dict(lddy=39), dict(dx=0), dict(lddx=39), dict(mean=0), dict(rstd=0), dict(mean=P + 1),
    dict(dgamma=P + 2), dict(dbeta=P + 1), dict(gamma=P + 1), dict(dy=P + 1), dict(dx=P + 1)])
def test_layernorm_backward_refusals(bad):
    assert bwd(**bad) == BAD, bad


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-2), dict(xt=5), dict(x=0), dict(ldx=39), dict(x=P + 1), dict(q=0), dict(e=0),
    dict(ldq=39), dict(lde=1)])
def test_checkpoint_refusals(bad):
    a = dict(rows=4, cols=40, x=P, ldx=40, xt=BF16, q=P, ldq=40, e=P, lde=2)
    a.update(bad)
    assert L.gemm_q8_save(a["rows"], a["cols"], a["x"], a["ldx"], a["xt"], a["q"], a["ldq"], a["e"], a["lde"],
                          stream=0) == BAD
    assert L.gemm_q8_restore(a["rows"], a["cols"], a["q"], a["ldq"], a["e"], a["lde"], a["x"], a["ldx"], a["xt"],
                             stream=0) == BAD


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(K=-1), dict(N=-1), dict(layout=2), dict(wt=4), dict(q=0), dict(e=0), dict(ldq=39), dict(lde=1),
    dict(dY=0), dict(lddy=7), dict(dY=P + 1), dict(dW=0), dict(ldw=7), dict(dW=P + 2), dict(base=P, ldbase=7),
    dict(base=P + 2, ldbase=8), dict(layout=L.GEMM_B_COL_MAJOR_NxK, ldw=39)])
def test_weight_grad_refusals(bad):
    assert wgrad(**bad) == BAD, bad


def test_extents_past_the_kernels_counters_are_unsupported():
    big = 1 << 31
    assert fwd(rows=big) == G.GEMM_ERR_UNSUPPORTED
    assert fwd(cols=big, ldx=big, ldy=big) == G.GEMM_ERR_UNSUPPORTED
    assert bwd(rows=big) == G.GEMM_ERR_UNSUPPORTED
    assert L.gemm_q8_save(big, 40, P, 40, BF16, P, 40, P, 2, stream=0) == G.GEMM_ERR_UNSUPPORTED
    assert wgrad(T=big) == G.GEMM_ERR_UNSUPPORTED
    assert wgrad(N=big, lddy=big, ldw=big) == G.GEMM_ERR_UNSUPPORTED


def test_empty_problems_are_noops():
    assert fwd(rows=0, x=0, y=0) == OK and fwd(cols=0, x=0, y=0) == OK
    assert bwd(cols=0, x=0, dy=0, dx=0) == OK
    assert bwd(rows=0, x=0, dy=0, dx=0, mean=0, rstd=0, dgamma=0, dbeta=0) == OK
    assert L.gemm_q8_save(0, 5, 0, 0, F32, 0, 0, 0, 0, stream=0) == OK
    assert L.gemm_q8_restore(5, 0, 0, 0, 0, 0, 0, 0, F32, stream=0) == OK
    assert wgrad(K=0, dW=0) == OK and wgrad(N=0, dW=0) == OK


def test_reference_checkpoint_by_hand():
    """The 64-bit reference itself, on blocks worked out by hand."""
    x = np.zeros((1, 96), np.float32)
    x[0, :4] = [127, -63.5, 0.5, 1.5]           # top = 127 * 2^0: E = 0, halves round to even
    x[0, 32:35] = [128, 127, -1]                # top past 127: E = 1
    x[0, 64] = np.inf
    q, e = R.q8_save(x)
    assert list(q[0, :4]) == [127, -64, 0, 2] and e[0, 0] == 127
    assert list(q[0, 32:35]) == [64, 64, 0] and e[0, 1] == 128
    assert e[0, 2] == 255 and not q[0, 64:].any()
    assert np.isnan(R.q8_values(q, e)[0, 64:]).all()


def test_reference_gradient_against_differences():
    """The reference's layer norm gradients against central differences of its
    forward pass, in 64 bits: with h = 1e-6 a difference is off by h^2 times a
    third derivative (order 1e-11 here) and 2^-52 / h = 2e-10 of rounding."""
    rng = np.random.default_rng(1)
    x, gamma, beta = rng.normal(size=(3, 17)), rng.normal(size=17), rng.normal(size=17)
    dy, eps, h = rng.normal(size=(3, 17)), 1e-5, 1e-6
    _, mean, rstd = R.ln_forward(x, gamma, beta, eps)
    dx, dg, db = R.ln_backward(x, mean, rstd, gamma, dy)

    def loss(x, gamma, beta):
        return float((R.ln_forward(x, gamma, beta, eps)[0] * dy).sum())
    for (i, j) in ((0, 0), (1, 5), (2, 16)):
        v = np.zeros_like(x)
        v[i, j] = h
        assert abs((loss(x + v, gamma, beta) - loss(x - v, gamma, beta)) / (2 * h) - dx[i, j]) < 1e-7
        w = np.zeros(17)
        w[j] = h
        assert abs((loss(x, gamma + w, beta) - loss(x, gamma - w, beta)) / (2 * h) - dg[j]) < 1e-7
        assert abs((loss(x, gamma, beta + w) - loss(x, gamma, beta - w)) / (2 * h) - db[j]) < 1e-7
