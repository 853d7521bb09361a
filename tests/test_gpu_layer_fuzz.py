"""Seeded random problems for the layer operators: sizes over their
logarithm, types, pitches, base offsets, absent parameters and outputs, each
against its 64-bit definition with the bounds of tests/layer_ref.py, and with
every output guarded."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import layer as L
from tests import layer_ref as R
from tests.test_gpu_layer import EPS, TYPES, Mat, _lib, activations, as_kind, done, vec, within  # noqa: F401

pytestmark = pytest.mark.gpu


def size(rng, lo, hi):
    v = int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))
    return max(lo, v // 8 * 8 if rng.random() < 0.5 and v >= 8 else v)


def place(rng):
    """(pad, offset) of a matrix in its buffer."""
    return (int(rng.choice([0, 0, 8, 16, 32, rng.integers(1, 40)])), int(rng.choice([0, 0, 0, 8, 16, rng.integers(1, 20)])))


def problem(rng, limit=400000):
    while True:
        rows, cols = size(rng, 1, 3000), size(rng, 1, 18000)
        if rows * cols <= limit:
            return rows, cols


@pytest.mark.parametrize("seed", range(60))
def test_layernorm_forward_random(seed):
    rng = np.random.default_rng(1000 + seed)
    rows, cols = problem(rng)
    xt, yt, pt = (str(rng.choice(["bf16", "f32"])) for _ in range(3))
    x = activations(rng, rows, cols, xt)
    gamma = as_kind(1 + 0.2 * rng.normal(size=cols), pt) if rng.random() < 0.8 else None
    beta = as_kind(0.2 * rng.normal(size=cols), pt) if rng.random() < 0.8 else None
    X, Y = Mat(rows, cols, xt, *place(rng), x), Mat(rows, cols, yt, *place(rng))
    stats = [Mat(1, rows, "f32", 0, int(rng.integers(0, 4))) if rng.random() < 0.7 else None for _ in range(2)]
    save = rng.random() < 0.6
    Q, E = Mat(rows, cols, "s8", *place(rng)), Mat(rows, -(-cols // 32), "u8", *place(rng))
    done(L.gemm_layernorm_forward(rows, cols, X.ptr, X.ld, TYPES[xt], vec(gamma, pt), vec(beta, pt), TYPES[pt], EPS,
                                  Y.ptr, Y.ld, TYPES[yt], *(s.ptr if s else None for s in stats),
                                  Q.ptr if save else None, Q.ld, E.ptr if save else None, E.ld))
    g, b = np.ones(cols) if gamma is None else gamma, np.zeros(cols) if beta is None else beta
    want = R.ln_forward(x, g, b, EPS)
    bound = R.ln_forward_bounds(x, g, b, EPS, yt)
    within(Y.host(), want[0], bound[0])
    for s, w, e in zip(stats, want[1:], bound[1:]):
        if s:
            within(s.host()[0], w, e)
            assert s.guarded()
    if save:
        q, e = R.q8_save(Y.host())
        assert np.array_equal(Q.host(), q) and np.array_equal(E.host(), e)
    assert all(a.guarded() for a in (X, Y, Q, E))


@pytest.mark.parametrize("seed", range(60))
def test_layernorm_backward_random(seed):
    rng = np.random.default_rng(2000 + seed)
    rows, cols = problem(rng)
    xt = str(rng.choice(["bf16", "f32", "q8"]))
    gt, pt = (str(rng.choice(["bf16", "f32"])) for _ in range(2))
    ot = str(rng.choice(["bf16", "f32"])) if xt == "q8" else xt
    x = activations(rng, rows, cols, "f32" if xt == "q8" else xt)
    X = Q = E = None
    if xt == "q8":
        q, e = R.q8_save(x)
        x = R.q8_values(q, e)
        Q, E = Mat(rows, cols, "s8", *place(rng), q), Mat(rows, -(-cols // 32), "u8", *place(rng), e)
    else:
        X = Mat(rows, cols, xt, *place(rng), x)
    gamma = as_kind(1 + 0.2 * rng.normal(size=cols), pt) if rng.random() < 0.8 else None
    g = np.ones(cols) if gamma is None else gamma
    _, m, s = R.ln_forward(x, g, 0, EPS)
    m, s = m.astype(np.float32), s.astype(np.float32)
    dy = rng.normal(size=(rows, cols)) * 10.0 ** rng.integers(-4, 3)
    dy[rng.random(rows) < 0.2] = 0
    dy = as_kind(dy, gt)
    D, O = Mat(rows, cols, gt, *place(rng), dy), Mat(rows, cols, ot, *place(rng))
    dg, db = (Mat(1, cols, "f32", 0, int(rng.integers(0, 4))) if rng.random() < 0.8 else None for _ in range(2))
    done(L.gemm_layernorm_backward(
        rows, cols, X.ptr if X else None, X.ld if X else 0, TYPES[ot], Q.ptr if Q else None, Q.ld if Q else 0,
        E.ptr if E else None, E.ld if E else 0, vec(gamma, pt), TYPES[pt], vec(m, "f32"), vec(s, "f32"), D.ptr, D.ld,
        TYPES[gt], O.ptr, O.ld, TYPES[ot], dg.ptr if dg else None, db.ptr if db else None))
    want = R.ln_backward(x, m, s, g, dy)
    bound = R.ln_backward_bounds(x, m, s, g, dy, ot)
    within(O.host(), want[0], bound[0])
    for a, w, e in ((dg, want[1], bound[1]), (db, want[2], bound[2])):
        if a:
            within(a.host()[0], w, e)
            assert a.guarded()
    assert D.guarded() and O.guarded()


@pytest.mark.parametrize("seed", range(60))
def test_weight_grad_random(seed):
    rng = np.random.default_rng(3000 + seed)
    while True:
        T, K, N = size(rng, 1, 5000), size(rng, 1, 3000), size(rng, 1, 3000)
        if T * K + T * N + K * N <= 1500000:
            break
    wt, nk = str(rng.choice(["f32", "bf16"])), bool(rng.random() < 0.5)
    q = rng.integers(-127, 128, size=(T, K)).astype(np.int8)
    e = rng.integers(115, 125, size=(T, -(-K // 32))).astype(np.uint8)
    dy = as_kind(rng.normal(size=(T, N)) * (rng.random((T, 1)) > 0.1), "bf16")
    shape = (N, K) if nk else (K, N)
    Q, E = Mat(T, K, "s8", *place(rng), q), Mat(T, -(-K // 32), "u8", *place(rng), e)
    D, W = Mat(T, N, "bf16", *place(rng), dy), Mat(*shape, wt, *place(rng))
    base = as_kind(rng.normal(size=shape), wt) if rng.random() < 0.6 else None
    B = None if base is None else W if rng.random() < 0.4 else Mat(*shape, wt, *place(rng))
    if B is not None:
        B.view.copy_(torch.from_numpy(base))
    done(L.gemm_q8_weight_grad(T, K, N, Q.ptr, Q.ld, E.ptr, E.ld, D.ptr, D.ld, B.ptr if B else None, B.ld if B else 0,
                               W.ptr, W.ld, L.GEMM_B_COL_MAJOR_NxK if nk else L.GEMM_B_ROW_MAJOR_KxN, TYPES[wt]))
    ref, mag = R.weight_grad(R.q8_values(q, e), dy, base, nk)
    within(W.host(), ref, R.weight_grad_bound(ref, mag, wt))
    assert all(a.guarded() for a in (Q, E, D, W))


@pytest.mark.parametrize("seed", range(40))
def test_checkpoint_random(seed):
    rng = np.random.default_rng(4000 + seed)
    rows, cols = problem(rng, 200000)
    kind, back = (str(rng.choice(["bf16", "f32"])) for _ in range(2))
    x = as_kind(rng.normal(size=(rows, cols)) * np.exp2(rng.integers(-140, 120, size=(rows, 1)).astype(np.float64)), kind)
    X, Q = Mat(rows, cols, kind, *place(rng), x), Mat(rows, cols, "s8", *place(rng))
    E, B = Mat(rows, -(-cols // 32), "u8", *place(rng)), Mat(rows, cols, back, *place(rng))
    done(L.gemm_q8_save(rows, cols, X.ptr, X.ld, TYPES[kind], Q.ptr, Q.ld, E.ptr, E.ld))
    done(L.gemm_q8_restore(rows, cols, Q.ptr, Q.ld, E.ptr, E.ld, B.ptr, B.ld, TYPES[back]))
    q, e = R.q8_save(x)
    assert np.array_equal(Q.host(), q) and np.array_equal(E.host(), e)
    assert np.array_equal(B.host().astype(np.float64), R.q8_values(q, e))
    assert all(a.guarded() for a in (X, Q, E, B))
