"""Dropout on the GPU against its definition (tests/gated_ref.py): what is kept
number for number, the values within their roundings; nothing outside the
matrices may change."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import layer as L
from tests import gated_ref as A
from tests.test_gpu_layer import TYPES, Mat, _lib, as_kind, done, within  # noqa: F401

pytestmark = pytest.mark.gpu
SEED, STEP = 0xFEDCBA9876543210, 2 ** 40 + 5

SHAPES = [(1, 1), (1, 4096), (2, 7), (3, 8), (4, 9), (5, 15), (6, 16), (9, 17), (40, 33), (129, 777), (64, 2048),
          (1000, 100), (7, 40003), (300, 250)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("xt,yt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
def test_forward_and_backward(rows, cols, xt, yt):
    rng = np.random.default_rng(rows + cols)
    x, r = as_kind(rng.normal(size=(rows, cols)), xt), as_kind(3 * rng.normal(size=(rows, cols)), yt)
    for p, pad, off in ((0.1, 0, 0), (0.5, 8, 8), (0.3, 3, 1)):
        X, Rm, Y = Mat(rows, cols, xt, pad, off, x), Mat(rows, cols, yt, pad, off, r), Mat(rows, cols, yt, pad, off)
        for res in (Rm, None):
            done(L.gemm_dropout_forward(rows, cols, X.ptr, X.ld, TYPES[xt], res and res.ptr, res.ld if res else 0,
                                        Y.ptr, Y.ld, TYPES[yt], p, SEED, STEP))
            within(Y.host(), *A.dropout(x, r if res else None, p, SEED, STEP, yt))
        assert np.array_equal(Y.host() != 0, A.keep(rows, cols, p, SEED, STEP) & (x != 0))
        # back: y's type in, x's out
        dy = as_kind(rng.normal(size=(rows, cols)), yt)
        D, dX = Mat(rows, cols, yt, pad, off, dy), Mat(rows, cols, xt, pad, off)
        done(L.gemm_dropout_backward(rows, cols, D.ptr, D.ld, TYPES[yt], dX.ptr, dX.ld, TYPES[xt], p, SEED, STEP))
        within(dX.host(), *A.dropout(dy, None, p, SEED, STEP, xt))
        assert np.array_equal(X.host(), x) and np.array_equal(Rm.host(), r)
        assert all(m.guarded() for m in (X, Rm, Y, D, dX))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("pads", [(0, 0), (3, 1)])
def test_in_place(kind, pads):
    """y over the residual, and over x; dx over dy."""
    rng = np.random.default_rng(4)
    x, r = (as_kind(rng.normal(size=(70, 203)), kind) for _ in range(2))
    X, Rm = Mat(70, 203, kind, *pads, x), Mat(70, 203, kind, *pads, r)
    t = TYPES[kind]
    done(L.gemm_dropout_forward(70, 203, X.ptr, X.ld, t, Rm.ptr, Rm.ld, Rm.ptr, Rm.ld, t, 0.25, 9, 1))
    within(Rm.host(), *A.dropout(x, r, 0.25, 9, 1, kind))
    done(L.gemm_dropout_forward(70, 203, X.ptr, X.ld, t, X.ptr, X.ld, X.ptr, X.ld, t, 0.25, 9, 2))
    within(X.host(), *A.dropout(x, x, 0.25, 9, 2, kind))
    X.view.copy_(torch.from_numpy(x))
    done(L.gemm_dropout_backward(70, 203, X.ptr, X.ld, t, X.ptr, X.ld, t, 0.25, 9, 3))
    within(X.host(), *A.dropout(x, None, 0.25, 9, 3, kind))
    assert X.guarded() and Rm.guarded()


def test_pitches_that_differ():
    """x, residual and y at pitches and offsets of their own, the mask the same."""
    rng = np.random.default_rng(5)
    x, r = as_kind(rng.normal(size=(37, 150)), "bf16"), as_kind(rng.normal(size=(37, 150)), "f32")
    for a, b, c in ((0, 1, 5), (8, 3, 0), (2, 0, 4)):
        X, Rm, Y = Mat(37, 150, "bf16", a, b, x), Mat(37, 150, "f32", b, c, r), Mat(37, 150, "f32", c, a)
        done(L.gemm_dropout_forward(37, 150, X.ptr, X.ld, TYPES["bf16"], Rm.ptr, Rm.ld, Y.ptr, Y.ld, TYPES["f32"], 0.4,
                                    3, 4))
        within(Y.host(), *A.dropout(x, r, 0.4, 3, 4, "f32"))
        assert Y.guarded()


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -17, 2.0 ** -16, 1 - 2.0 ** -16, 0.9999999])
def test_ends_of_p(p):
    x = as_kind(np.random.default_rng(6).normal(size=(64, 1000)), "f32")
    X, Y = Mat(64, 1000, "f32", fill=x), Mat(64, 1000, "f32")
    done(L.gemm_dropout_forward(64, 1000, X.ptr, 1000, 0, X.ptr, 1000, Y.ptr, 1000, 0, p, 11, 12))
    within(Y.host(), *A.dropout(x, x, p, 11, 12, "f32"))
    done(L.gemm_dropout_backward(64, 1000, X.ptr, 1000, 0, Y.ptr, 1000, 0, p, 11, 12))
    assert np.array_equal(Y.host() != 0, A.keep(64, 1000, p, 11, 12) & (x != 0))


def test_dropped_values_contribute_nothing():
    """A dropped NaN or infinity leaves the residual as it is, bit for bit."""
    rng = np.random.default_rng(8)
    x, r = as_kind(np.full((50, 90), np.nan), "bf16"), as_kind(rng.normal(size=(50, 90)), "bf16")
    x[25:] = np.inf
    X, Rm, Y = Mat(50, 90, "bf16", fill=x), Mat(50, 90, "bf16", fill=r), Mat(50, 90, "bf16")
    done(L.gemm_dropout_forward(50, 90, X.ptr, 90, 1, Rm.ptr, 90, Y.ptr, 90, 1, 0.5, 1, 2))
    k, y = A.keep(50, 90, 0.5, 1, 2), Y.host()
    assert np.array_equal(y[~k], r[~k]) and not np.isfinite(y[k]).any()


def test_steps_on_the_device_and_in_graphs():
    """The device's word is added to the step modulo 2^64 when the kernel runs:
    a replayed graph that counts it up draws anew each time."""
    x = as_kind(np.random.default_rng(9).normal(size=(33, 64)), "f32")
    X, Y = Mat(33, 64, "f32", fill=x), Mat(33, 64, "f32")
    word = torch.tensor([2 ** 62], dtype=torch.int64, device="cuda")
    first = 2 ** 64 - 2 ** 62 - 1

    def call(stream=None):
        return L.gemm_dropout_backward(33, 64, X.ptr, 64, 0, Y.ptr, 64, 0, 0.5, 21, first, word, stream=stream)
    done(call())
    within(Y.host(), *A.dropout(x, None, 0.5, 21, 2 ** 64 - 1, "f32"))
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=st):
        word.add_(1)
        status = call(st)
    assert status == 0
    for n in range(3):
        graph.replay()
        torch.cuda.synchronize()
        within(Y.host(), *A.dropout(x, None, 0.5, 21, n, "f32"))
