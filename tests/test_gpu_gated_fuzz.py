"""Seeded random problems for the gated feed-forward and dropout calls: sizes
over their logarithm, layouts, activations, pitches and base offsets of every
matrix apart, absent outputs, in place or not; each against its 64-bit
definition, with every output guarded."""
import numpy as np
import pytest

from paper_2512_13282_gb300 import layer as L
from tests import gated_ref as A
from tests.test_gpu_dropout import TYPES  # noqa: F401
from tests.test_gpu_gated import ACT, KN, NK, bf, check_backward, gate_inputs
from tests.test_gpu_layer import Mat, _lib, as_kind, done, within  # noqa: F401
from tests.test_gpu_layer_fuzz import place, size

pytestmark = pytest.mark.gpu


def problem(rng, limit):
    while True:
        t, k, f = size(rng, 1, 2500), size(rng, 1, 3000), size(rng, 1, 3000)
        if t * k * f <= limit:
            return t, k, f


def weight(rng, K, F, layout):
    w = bf(rng.normal(size=(K, F)) / K ** 0.5)
    v = w if layout == KN else w.T
    return w, Mat(*v.shape, "bf16", *place(rng), v)


@pytest.mark.parametrize("seed", range(60))
def test_forward_random(seed):
    rng = np.random.default_rng(3000 + seed)
    T, K, F = problem(rng, 4e8)
    layout, act = int(rng.choice([KN, NK])), str(rng.choice(A.ACTS))
    x = bf(rng.normal(size=(T, K)) * float(rng.choice([0.1, 1, 5])))
    (wg, Wg), (wu, Wu) = weight(rng, K, F, layout), weight(rng, K, F, layout)
    X, out = Mat(T, K, "bf16", *place(rng), x), [Mat(T, F, "bf16", *place(rng)) for _ in range(3)]
    keep = rng.random() < 0.6
    kept = [a for m in out[1:] for a in ((m.ptr, m.ld) if keep else (None, 0))]
    done(L.gemm_gated_forward(T, K, F, X.ptr, X.ld, Wg.ptr, Wg.ld, Wu.ptr, Wu.ld, layout, ACT[act], out[0].ptr,
                              out[0].ld, *kept))
    for m, (want, bound) in list(zip(out, A.forward(x, wg, wu, act)))[:3 if keep else 1]:
        within(m.host(), want, bound)
    assert all(m.guarded() for m in out + [X, Wg, Wu])


@pytest.mark.parametrize("seed", range(60))
def test_backward_random(seed):
    rng = np.random.default_rng(4000 + seed)
    T, N, F = problem(rng, 4e8)
    act, held, product = str(rng.choice(A.ACTS)), rng.random() < 0.7, rng.random() < 0.7
    g, u = gate_inputs(rng, T, F)
    Gm, U = Mat(T, F, "bf16", *place(rng), g), Mat(T, F, "bf16", *place(rng), u)
    dG = Gm if rng.random() < 0.3 else Mat(T, F, "bf16", *place(rng))
    dU = U if rng.random() < 0.3 else Mat(T, F, "bf16", *place(rng))
    Q, E = Mat(T, F, "s8", *place(rng)), Mat(T, -(-F // 32), "u8", *place(rng))
    rest = (Gm.ptr, Gm.ld, U.ptr, U.ld, ACT[act], dG.ptr, dG.ld, dU.ptr, dU.ld, Q.ptr if held else None, Q.ld,
            E.ptr if held else None, E.ld)
    if product:
        layout = int(rng.choice([KN, NK]))
        d = bf(1e-2 * rng.normal(size=(T, N)))
        wdT, Wd = weight(rng, F, N, layout)            # Wd is F x N: KxN has its rows F
        D = Mat(T, N, "bf16", *place(rng), d)
        done(L.gemm_gated_down_backward(T, N, F, D.ptr, D.ld, Wd.ptr, Wd.ld, layout, *rest))
        dh, edh = A.product(d, wdT.T)
    else:
        dh, edh = bf(1e-2 * rng.normal(size=(T, F))), 0
        D = Mat(T, F, "bf16", *place(rng), dh)
        done(L.gemm_gated_backward(T, F, D.ptr, D.ld, *rest))
    assert all(m.guarded() for m in (Gm, U, dG, dU, Q, E, D))
    check_backward(dh, edh, g, u, act, [dG.host(), dU.host()], (Q.host(), E.host()) if held else None)


@pytest.mark.parametrize("seed", range(60))
def test_dropout_random(seed):
    rng = np.random.default_rng(5000 + seed)
    while True:
        rows, cols = size(rng, 1, 3000), size(rng, 1, 18000)
        if rows * cols <= 400000:
            break
    xt, yt = (str(rng.choice(["bf16", "f32"])) for _ in range(2))
    p, key, step = float(rng.random()), int(rng.integers(2 ** 63)) * 2 + 1, int(rng.integers(2 ** 63))
    x = as_kind(rng.normal(size=(rows, cols)), xt)
    r = as_kind(rng.normal(size=(rows, cols)), yt) if rng.random() < 0.6 else None
    X, Rm = Mat(rows, cols, xt, *place(rng), x), Mat(rows, cols, yt, *place(rng), r)
    Y = Rm if r is not None and rng.random() < 0.3 else Mat(rows, cols, yt, *place(rng))
    done(L.gemm_dropout_forward(rows, cols, X.ptr, X.ld, TYPES[xt], Rm.ptr if r is not None else None, Rm.ld, Y.ptr,
                                Y.ld, TYPES[yt], p, key, step))
    within(Y.host(), *A.dropout(x, r, p, key, step, yt))
    assert all(m.guarded() for m in (X, Rm, Y))
