"""Host-side checks of the gated feed-forward and dropout calls that need no
GPU: refusals before the device is touched, no-ops, and the references
themselves against differences and published numbers."""
import numpy as np
import pytest

from paper_2512_13282_gb300 import build as B
from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from tests import gated_ref as A
from tests import layer_ref as R

P = 0x1000  # an aligned address that is never dereferenced: validation fails first
F32, BF16 = L.GEMM_TYPE_F32, L.GEMM_TYPE_BF16
KN, NK = L.GEMM_B_ROW_MAJOR_KxN, L.GEMM_B_COL_MAJOR_NxK
BAD, OK, NO = G.GEMM_ERR_INVALID_ARG, G.GEMM_OK, G.GEMM_ERR_UNSUPPORTED


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return L.library()


def fwd(T=4, K=40, F=24, X=P, ldx=40, Wg=P, ldwg=24, Wu=P, ldwu=24, layout=KN, act=0, H=P, ldh=24, Gm=0, ldg=0, U=0,
        ldu=0):
    return L.gemm_gated_forward(T, K, F, X, ldx, Wg, ldwg, Wu, ldwu, layout, act, H, ldh, Gm, ldg, U, ldu, stream=0)


GRAD = dict(Gm=P, ldg=24, U=P, ldu=24, act=0, dG=P, lddg=24, dU=P, lddu=24, q=0, ldq=0, e=0, lde=0)


def bwd(T=4, F=24, dH=P, lddh=24, **rest):
    return L.gemm_gated_backward(T, F, dH, lddh, *{**GRAD, **rest}.values(), stream=0)


def down(T=4, N=40, F=24, dO=P, lddo=40, Wd=P, ldwd=40, layout=KN, **rest):
    return L.gemm_gated_down_backward(T, N, F, dO, lddo, Wd, ldwd, layout, *{**GRAD, **rest}.values(), stream=0)


def drop(rows=4, cols=24, x=P, ldx=24, xt=BF16, res=P, ldr=24, y=P, ldy=24, yt=BF16, p=0.1, seed=1, step=2, dev=0):
    return L.gemm_dropout_forward(rows, cols, x, ldx, xt, res, ldr, y, ldy, yt, p, seed, step, dev, stream=0)


def back(rows=4, cols=24, x=P, ldx=24, xt=BF16, y=P, ldy=24, yt=BF16, p=0.1, seed=1, step=2, dev=0):
    return L.gemm_dropout_backward(rows, cols, x, ldx, xt, y, ldy, yt, p, seed, step, dev, stream=0)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(K=-1), dict(F=-1), dict(layout=2), dict(act=4), dict(act=-1), dict(X=0), dict(ldx=39), dict(Wg=0),
    dict(Wu=0), dict(ldwg=23), dict(ldwu=23), dict(layout=NK, ldwg=39, ldwu=40), dict(layout=NK, ldwg=40, ldwu=39),
    dict(H=0), dict(ldh=23), dict(Gm=P, ldg=24), dict(U=P, ldu=24), dict(Gm=P, ldg=23, U=P, ldu=24),
    dict(Gm=P, ldg=24, U=P, ldu=23), dict(X=P + 1), dict(Wg=P + 1), dict(Wu=P + 1), dict(H=P + 1),
    dict(Gm=P + 1, ldg=24, U=P, ldu=24)])
def test_gated_forward_refusals(bad):
    assert fwd(**bad) == BAD, bad


SHARED = [dict(T=-1), dict(F=-1), dict(act=4), dict(act=-1), dict(Gm=0), dict(U=0), dict(dG=0), dict(dU=0),
          dict(ldg=23), dict(ldu=23), dict(lddg=23), dict(lddu=23), dict(Gm=P + 1), dict(U=P + 1), dict(dG=P + 1),
          dict(dU=P + 1), dict(q=P, ldq=24), dict(e=P, lde=1), dict(q=P, ldq=23, e=P, lde=1),
          dict(q=P, ldq=24, e=P, lde=0)]


@pytest.mark.parametrize("bad", SHARED + [dict(dH=0), dict(dH=P + 1), dict(lddh=23)])
def test_gated_backward_refusals(bad):
    assert bwd(**bad) == BAD, bad


@pytest.mark.parametrize("bad", SHARED + [
    dict(N=-1), dict(layout=-1), dict(dO=0), dict(dO=P + 1), dict(lddo=39), dict(Wd=0), dict(Wd=P + 1), dict(ldwd=39),
    dict(layout=NK, ldwd=23)])
def test_gated_down_backward_refusals(bad):
    assert down(**bad) == BAD, bad


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(cols=-1), dict(xt=2), dict(yt=-1), dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(x=0),
    dict(y=0), dict(ldx=23), dict(ldy=23), dict(x=P + 1), dict(y=P + 2, yt=F32), dict(dev=P + 4)])
def test_dropout_refusals(bad):
    assert drop(**bad) == BAD and back(**bad) == BAD, bad
    assert drop(res=P, ldr=23) == BAD and drop(res=P + 1) == BAD


def test_extents_past_the_kernels_counters_are_unsupported():
    big = 1 << 31
    assert fwd(T=big) == NO and fwd(K=big, ldx=big) == NO and fwd(F=big, ldwg=big, ldwu=big, ldh=big) == NO
    assert bwd(T=big) == NO
    assert down(T=big) == NO and down(N=big, lddo=big, ldwd=big) == NO
    assert drop(rows=big) == NO and back(cols=big, ldx=big, ldy=big) == NO


def test_empty_problems_are_noops():
    assert fwd(T=0, X=0, H=0) == OK and fwd(F=0, Wg=0, H=0) == OK
    assert bwd(T=0, dH=0) == OK and bwd(F=0, dG=0) == OK
    assert down(T=0, dO=0) == OK and down(F=0, Wd=0) == OK
    assert drop(rows=0, x=0, y=0) == OK and back(cols=0, x=0) == OK


@pytest.mark.parametrize("kind", A.ACTS)
def test_reference_slope_against_differences(kind):
    """Central differences with h = 1e-6: off by h^2 times a third derivative
    and 2^-53 |g| / h of rounding; relu away from its corner."""
    g = np.linspace(-9, 9, 1801) + 1e-3
    h = 1e-6
    slope = (A.act(g + h, kind)[0] - A.act(g - h, kind)[0]) / (2 * h)
    assert np.abs(slope - A.act(g, kind)[1]).max() < 1e-8
    assert np.abs(A.act(g, kind)[1]).max() < A.TOP_SLOPE


def test_reference_gate_gradient_against_differences():
    rng = np.random.default_rng(3)
    g, u, dh = (rng.normal(size=(3, 5)) for _ in range(3))
    (dg, _), (du, _), (h, _) = A.backward(dh, 0, g, u, "silu")
    step = 1e-6
    for i, j in ((0, 0), (2, 3)):
        v = np.zeros_like(g)
        v[i, j] = step

        def loss(g, u):
            return float((A.act(g, "silu")[0] * u * dh).sum())
        assert abs((loss(g + v, u) - loss(g - v, u)) / (2 * step) - dg[i, j]) < 1e-8
        assert abs((loss(g, u + v) - loss(g, u - v)) / (2 * step) - du[i, j]) < 1e-8
    assert np.array_equal(h, A.act(g, "silu")[0] * u)


def test_reference_generator():
    """The known answers published with the generator: counter and key of
    zeros, and of ones throughout."""
    assert [int(v) for v in A.philox([[0]] * 4, (0, 0))[:, 0]] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert [int(v) for v in A.philox([[ones]] * 4, (ones, ones))[:, 0]] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_reference_keep():
    """The share kept is 1 - P within five standard deviations; neighbouring
    columns, rows and steps draw apart; nothing is dropped at 0, all at 1."""
    n = 400 * 1000
    for p in (0.1, 0.5):
        k = A.keep(400, 1000, p, 7, 3)
        P = A.threshold(p) / 65536
        assert abs(k.mean() - (1 - P)) < 5 * np.sqrt(P * (1 - P) / n)
    a, b = A.keep(64, 96, 0.5, 7, 3), A.keep(64, 96, 0.5, 7, 4)
    assert (a != b).any() and (a[0] != a[1]).any() and (a[:, :8] != a[:, 8:16]).any()
    assert A.keep(3, 9, 0.0, 1, 1).all() and not A.keep(3, 9, 1.0, 1, 1).any()


def test_reference_checkpoint_check():
    """held_ok takes a block's own checkpoint and refuses one a step or an exponent off."""
    h = np.random.default_rng(1).normal(size=(2, 70))
    q, e = R.q8_save(h.astype(np.float32))
    err = 2.0 ** -20 * np.abs(h)
    assert A.held_ok(q, e, h, err)
    bad = q.copy()
    bad[1, 69] += 1 if bad[1, 69] < 100 else -1
    assert not A.held_ok(bad, e, h, err)
    bad = e.copy()
    bad[0, 0] += 1
    assert not A.held_ok((q / 2).astype(np.int8), bad, h, err)
