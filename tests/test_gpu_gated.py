"""The gated feed-forward block's calls on the GPU against their definitions in
64 bits (tests/gated_ref.py), within bounds derived from their float32
operations.  Every output lies in a guarded buffer: nothing outside its matrix
may change, and inputs stay as they are."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from tests import gated_ref as A
from tests.test_gpu_layer import Mat, _lib, as_kind, done, within  # noqa: F401

pytestmark = pytest.mark.gpu

ACT = {"silu": L.GEMM_ACT_SILU, "gelu": L.GEMM_ACT_GELU, "gelu_tanh": L.GEMM_ACT_GELU_TANH, "relu": L.GEMM_ACT_RELU}
KN, NK = L.GEMM_B_ROW_MAJOR_KxN, L.GEMM_B_COL_MAJOR_NxK
NAMES = {KN: "KxN", NK: "NxK"}


def bf(x):
    return as_kind(x, "bf16")


def weight(w, layout, pad=0, off=0):
    """A K x F weight on the device in a layout."""
    w = w if layout == KN else w.T
    return Mat(*w.shape, "bf16", pad, off, w)


def run_forward(x, wg, wu, act, layout, pad=0, off=0, save=True, stream=None):
    (T, K), F = x.shape, wg.shape[1]
    X, Wg, Wu = Mat(T, K, "bf16", pad, off, x), weight(wg, layout, pad, off), weight(wu, layout, pad, off)
    out = [Mat(T, F, "bf16", pad, off) for _ in range(3 if save else 1)]
    kept = [a for m in out[1:] for a in (m.ptr, m.ld)]
    done(L.gemm_gated_forward(T, K, F, X.ptr, X.ld, Wg.ptr, Wg.ld, Wu.ptr, Wu.ld, layout, ACT[act], out[0].ptr,
                              out[0].ld, *kept, stream=stream))
    assert all(m.guarded() for m in out + [X, Wg, Wu])
    return [m.host() for m in out]


def check_forward(T, K, F, act, layout, pad=0, off=0, save=True, scale=1.0):
    rng = np.random.default_rng(T * 7 + K * 3 + F)
    x = bf(scale * rng.normal(size=(T, K)))
    wg, wu = (bf(rng.normal(size=(K, F)) / K ** 0.5) for _ in range(2))
    got = run_forward(x, wg, wu, act, layout, pad, off, save)
    for g, (want, bound) in zip(got, A.forward(x, wg, wu, act)):
        within(g, want, bound)


# one token and few, around every tile's edge, odd and even widths, one value
FORWARD = [(1, 1, 1), (1, 64, 64), (1, 4096, 1000), (2, 777, 129), (3, 72, 65), (8, 512, 2048), (15, 200, 96),
           (16, 1500, 192), (17, 64, 31), (33, 328, 777), (48, 1024, 1376), (64, 130, 512), (65, 96, 64), (100, 4096, 256),
           (127, 64, 1501), (128, 520, 640), (129, 256, 200), (200, 1000, 136), (256, 64, 384), (300, 777, 301),
           (513, 192, 264), (1000, 128, 130), (129, 4096, 264), (600, 2048, 1504), (2100, 256, 2000), (20000, 3, 5),
           (9000, 8, 8)]


@pytest.mark.parametrize("layout", [KN, NK], ids=NAMES.get)
@pytest.mark.parametrize("T,K,F", FORWARD)
def test_forward(T, K, F, layout):
    act = A.ACTS[(T + K + F) % 4]
    check_forward(T, K, F, act, layout)
    check_forward(T, K, F, act, layout, 8, 8, False)
    check_forward(T, K, F, act, layout, 3, 1, True)


@pytest.mark.parametrize("act", A.ACTS)
@pytest.mark.parametrize("T", [1, 40, 300])
def test_forward_activations(T, act):
    """Sums from far below to far above zero: the activations' ends."""
    check_forward(T, 64, 200, act, KN, scale=12.0)


def test_forward_of_nothing_to_sum():
    H, G_, U = (Mat(5, 70, "bf16", 3, 1) for _ in range(3))
    done(L.gemm_gated_forward(5, 0, 70, None, 0, None, 0, None, 0, KN, 0, H.ptr, H.ld, G_.ptr, G_.ld, U.ptr, U.ld))
    assert all((m.host() == 0).all() and m.guarded() for m in (H, G_, U))


@pytest.mark.parametrize("T", [1, 20, 300])
@pytest.mark.parametrize("layout", [KN, NK], ids=NAMES.get)
def test_forward_of_halves_of_one_matrix(T, layout):
    """Wg and Wu halves of one weight, G and U of one matrix; F odd, so that the
    second halves start off 16 bytes."""
    K, F = 136, 101
    rng = np.random.default_rng(T)
    x, w = bf(rng.normal(size=(T, K))), bf(rng.normal(size=(K, 2 * F)) / 12)
    X, W, GU, H = Mat(T, K, "bf16", fill=x), weight(w, layout), Mat(T, 2 * F, "bf16"), Mat(T, F, "bf16")
    second = 2 * F * (1 if layout == KN else W.ld)
    done(L.gemm_gated_forward(T, K, F, X.ptr, K, W.ptr, W.ld, W.ptr + second, W.ld, layout, ACT["silu"], H.ptr, F,
                              GU.ptr, 2 * F, GU.ptr + 2 * F, 2 * F))
    want = A.forward(x, w[:, :F], w[:, F:], "silu")
    within(H.host(), *want[0])
    within(GU.host(), *(np.hstack(v) for v in zip(*want[1:])))
    assert GU.guarded() and H.guarded()


@pytest.mark.parametrize("T", [1, 30, 200])
def test_forward_of_infinite_and_nan_tokens(T):
    """A token with a NaN or an infinity spoils its own row and no other."""
    K, F = 96, 130
    rng = np.random.default_rng(T)
    x, wg, wu = bf(rng.normal(size=(T, K))), bf(rng.normal(size=(K, F))), bf(rng.normal(size=(K, F)))
    bad = x.copy()
    bad[0, 3] = np.nan
    if T > 2:
        bad[T // 2, 95] = np.inf
    for layout in (KN, NK):
        got, clean = run_forward(bad, wg, wu, "silu", layout), run_forward(x, wg, wu, "silu", layout)
        assert all(np.isnan(a[0]).all() for a in got)
        keep = np.ones(T, bool)
        keep[[0, T // 2]] = False
        for a, b in zip(got, clean):
            assert np.array_equal(a[keep], b[keep])
        if T > 2:
            assert not np.isfinite(got[1][T // 2]).any()


# ------------------------------------------------------------------- backward

def gate_inputs(rng, T, F):
    g, u = bf(1.5 * rng.normal(size=(T, F))), bf(rng.normal(size=(T, F)))
    if F > 2:
        g[0, :2] = [30.0, -30.0]
        u[0, 2] = 0.0
    return g, u


def run_backward(g, u, act, held, call, pad=0, off=0, in_place=False):
    """call(the arguments behind dH's) -> [dG, dU] and (q, e)."""
    T, F = g.shape
    Gm, U = Mat(T, F, "bf16", pad, off, g), Mat(T, F, "bf16", pad, off, u)
    dG, dU = (Gm, U) if in_place else (Mat(T, F, "bf16", pad, off), Mat(T, F, "bf16", pad, off))
    Q, E = Mat(T, F, "s8", pad, off), Mat(T, -(-F // 32), "u8", pad, off)
    ck = (Q.ptr, Q.ld, E.ptr, E.ld) if held else (None, 0, None, 0)
    done(call(Gm.ptr, Gm.ld, U.ptr, U.ld, ACT[act], dG.ptr, dG.ld, dU.ptr, dU.ld, *ck))
    assert all(m.guarded() for m in (Gm, U, dG, dU, Q, E))
    if not in_place:
        assert np.array_equal(Gm.host(), g, equal_nan=True) and np.array_equal(U.host(), u)
    return [dG.host(), dU.host()], ((Q.host(), E.host()) if held else None)


def check_backward(dh, edh, g, u, act, got, ck):
    dg, du, h = A.backward(dh, edh, g, u, act)
    within(got[0], *dg)
    within(got[1], *du)
    if ck:
        assert A.held_ok(*ck, *h)


def gate_grad(T, F, act, pad=0, off=0, held=True, in_place=False):
    rng = np.random.default_rng(T * 11 + F)
    g, u = gate_inputs(rng, T, F)
    dh = bf(1e-2 * rng.normal(size=(T, F)))
    D = Mat(T, F, "bf16", pad, off, dh)
    got, ck = run_backward(g, u, act, held, lambda *a: L.gemm_gated_backward(T, F, D.ptr, D.ld, *a), pad, off, in_place)
    check_backward(dh, 0, g, u, act, got, ck)


BACKWARD = [(1, 1), (1, 11008), (2, 31), (3, 32), (5, 33), (7, 64), (40, 777), (129, 1501), (64, 2048), (1000, 96),
            (33, 4096), (2, 40008), (2000, 1001), (700, 4104)]


@pytest.mark.parametrize("T,F", BACKWARD)
@pytest.mark.parametrize("act", A.ACTS)
def test_backward(T, F, act):
    gate_grad(T, F, act)
    gate_grad(T, F, act, 8, 8, False)
    gate_grad(T, F, act, 16, 16, True, True)
    gate_grad(T, F, act, 3, 1)
    gate_grad(T, F, act, 5, 7, True, True)


DOWN = [(1, 1, 1), (1, 4096, 640), (3, 777, 33), (16, 64, 64), (40, 328, 200), (100, 1000, 129), (128, 128, 256),
        (129, 96, 777), (256, 512, 320), (300, 777, 301), (513, 64, 264), (1000, 136, 130), (70, 2048, 1376),
        (300, 4096, 520), (600, 2048, 1504), (130, 3000, 1000), (2100, 256, 2008), (90, 100, 32), (300, 64, 96),
        (1000, 520, 480), (2100, 256, 2016), (129, 4096, 544), (300, 4096, 352), (20000, 3, 5), (9000, 8, 8)]


def down_grad(T, N, F, act, layout, pad=0, off=0, held=True, in_place=False):
    rng = np.random.default_rng(T * 5 + N * 3 + F)
    g, u = gate_inputs(rng, T, F)
    d, wd = bf(1e-2 * rng.normal(size=(T, N))), bf(rng.normal(size=(F, N)) / N ** 0.5)
    D, W = Mat(T, N, "bf16", pad, off, d), weight(wd, layout, pad, off)
    got, ck = run_backward(
        g, u, act, held, lambda *a: L.gemm_gated_down_backward(T, N, F, D.ptr, D.ld, W.ptr, W.ld, layout, *a), pad, off,
        in_place)
    assert D.guarded() and W.guarded()
    check_backward(*A.product(d, wd.T), g, u, act, got, ck)


@pytest.mark.parametrize("layout", [KN, NK], ids=NAMES.get)
@pytest.mark.parametrize("T,N,F", DOWN)
def test_down_backward(T, N, F, layout):
    act = A.ACTS[(T + N + F) % 4]
    down_grad(T, N, F, act, layout)
    down_grad(T, N, F, act, layout, 8, 8, False)
    down_grad(T, N, F, act, layout, 16, 16, True, True)
    down_grad(T, N, F, act, layout, 3, 1)
    down_grad(T, N, F, act, layout, 5, 7, True, True)


@pytest.mark.parametrize("act", A.ACTS)
def test_down_backward_activations(act):
    down_grad(300, 64, 200, act, KN)


def test_down_backward_of_nothing_to_sum():
    """dH is zero, and the checkpoint is H's all the same."""
    rng = np.random.default_rng(2)
    g, u = gate_inputs(rng, 9, 70)
    got, ck = run_backward(g, u, "gelu", True, lambda *a: L.gemm_gated_down_backward(9, 0, 70, None, 0, None, 0, KN, *a))
    assert not got[0].any() and not got[1].any()
    check_backward(np.zeros((9, 70)), 0, g, u, "gelu", got, ck)


@pytest.mark.parametrize("act", A.ACTS)
def test_gradients_where_activations_end(act):
    """Gates from the smallest to the largest bf16 numbers: finite products stay
    finite, NaN stays NaN, an infinite gate's block of the checkpoint is NaN."""
    top = 3.3895e38
    g = bf(np.array([[0.0, -0.0, 1e-40, -1e-40, 1e-30, -1e-30, 20, -20, 88, -88, 100, -100, 1e4, -1e4, 1e13, -1e13,
                      1e19, -1e19, 1e30, -1e30, top, -top, 0.5, -0.5]]))
    u, dh = np.ones_like(g), bf(np.full_like(g, 0.5))
    D = Mat(*g.shape, "bf16", fill=dh)
    got, ck = run_backward(g, u, act, True, lambda *a: L.gemm_gated_backward(1, g.shape[1], D.ptr, D.ld, *a))
    with np.errstate(over="ignore", invalid="ignore"):
        a, s = A.act(np.clip(g.astype(np.float64), -1e6, 1e6), act)   # past that the ends' own values
    a = np.where(g > 1e6, g, np.where(g < -1e6, 0, a))
    assert np.isfinite(got[0]).all()
    within(got[0], 0.5 * s, 0.5 * A.ACT + 2.0 ** -8 * np.abs(0.5 * s))
    within(got[1], 0.5 * a, 0.5 * A.ACT * np.abs(g) + 2.0 ** -8 * np.abs(0.5 * a) + 2.0 ** -133)
    for special in (np.nan, np.inf):
        g[0, 5] = special
        got, ck = run_backward(g, u, act, True, lambda *a: L.gemm_gated_backward(1, g.shape[1], D.ptr, D.ld, *a))
        assert not np.isfinite(got[1][0, 5]) and ck[1][0, 0] == 255 and not ck[0].any()
        assert np.isnan(got[0][0, 5]) or special == np.inf
        keep = np.arange(g.shape[1]) != 5
        assert np.isfinite(got[0][0, keep]).all()
