"""The gate of far negative values, where act(g) is small but still a normal
number: its relative accuracy, in every kernel that takes it.

Bound.  act(g) and its slope are products of an exponential of x -- x = |g|, g^2 / 2
or 2 |z| -- and factors near one.  Results that are normal numbers have x <= 92: the
argument's roundings (six at most) give 6 * 92 * 2^-24 = 2^-14.9 of the
exponential, its own error (2 + 1.2 x) 2^-23 < 2^-16, its place below the normal
numbers 2^-150 of 2^-133, the normal distribution's tail 2^-20 and the other
operations a few 2^-24: together below 2^-14.  A slope's two terms are at most 2.1
times their sum for g <= -3.  Then the result's rounding to bf16."""
import numpy as np
import pytest

from paper_2512_13282_gb300 import layer as L
from tests import gated_ref as A
from tests.test_gpu_gated import ACT, KN, bf
from tests.test_gpu_layer import Mat, _lib, done  # noqa: F401

pytestmark = pytest.mark.gpu

REL_ACT = 2.0 ** -14 + 2.0 ** -8 * (1 + 2.0 ** -14)
REL_SLOPE = 2.1 * 2.0 ** -14 + 2.0 ** -8 * (1 + 2.0 ** -12)
KINDS = ["silu", "gelu", "gelu_tanh"]


def gates(kind):
    """All bf16 numbers from -3 down with |act| >= 2^-126."""
    g = (np.arange(0xC040, 0xC2C8, dtype=np.uint32) << 16).view(np.float32)   # -3 .. -100
    assert g[0] == -3 and g[-1] < -99
    return g[np.abs(A.act(g, kind)[0]) >= 2.0 ** -126]


def near(got, want, rel):
    assert (np.abs(got - want) <= rel * np.abs(want)).all(), np.abs(got / want - 1).max()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("product,T", [(False, 300), (True, 300), (True, 60)])
def test_gradient(kind, product, T):
    """dH = 1 and U = 1 leave the slope in dG and the activation in dU."""
    g = gates(kind)
    F = len(g)
    G, ones = Mat(T, F, "bf16", fill=bf(np.broadcast_to(g, (T, F)))), np.ones((T, F), np.float32)
    U, dG, dU = Mat(T, F, "bf16", fill=ones), Mat(T, F, "bf16"), Mat(T, F, "bf16")
    rest = (G.ptr, F, U.ptr, F, ACT[kind], dG.ptr, F, dU.ptr, F)
    if product:
        D, W = Mat(T, 1, "bf16", fill=ones[:, :1]), Mat(F, 1, "bf16", fill=np.ones((F, 1), np.float32))
        done(L.gemm_gated_down_backward(T, 1, F, D.ptr, 1, W.ptr, 1, KN, *rest))
    else:
        D = Mat(T, F, "bf16", fill=ones)
        done(L.gemm_gated_backward(T, F, D.ptr, F, *rest))
    a, s = A.act(g, kind)
    near(dU.host().astype(np.float64), np.broadcast_to(a, (T, F)), REL_ACT)
    near(dG.host().astype(np.float64), np.broadcast_to(s, (T, F)), REL_SLOPE)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [60, 300])
def test_forward(kind, T):
    """X = 1, Wg the gates, Wu = 1."""
    g = gates(kind)
    F = len(g)
    X, Wg = Mat(T, 1, "bf16", fill=np.ones((T, 1), np.float32)), Mat(1, F, "bf16", fill=bf(g[None]))
    Wu, H = Mat(1, F, "bf16", fill=np.ones((1, F), np.float32)), Mat(T, F, "bf16")
    done(L.gemm_gated_forward(T, 1, F, X.ptr, 1, Wg.ptr, F, Wu.ptr, F, KN, ACT[kind], H.ptr, F))
    near(H.host().astype(np.float64), np.broadcast_to(A.act(g, kind)[0], (T, F)), REL_ACT)
