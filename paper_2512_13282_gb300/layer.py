"""ctypes binding of the C ABI in ``include/gb300_layer.h`` -- the operators
around a projection GEMM in training (layer norm, 8-bit activation
checkpoints, the weight gradient, the gated feed-forward block's gate and its
gradient, dropout); argument marshalling only.

Names, argument order and conventions are the header's, and those of
``gemm``: pointer arguments accept an integer device address, a CUDA
``torch.Tensor`` or ``None``; ``stream`` an integer, a ``torch.cuda.Stream``
or ``None`` (torch's current stream).  Each call returns a status; ``check``
raises ``GemmError`` for one that is not ``GEMM_OK``.
"""
from __future__ import annotations

import ctypes

from . import gemm as _gemm
from .gemm import (GEMM_B_COL_MAJOR_NxK, GEMM_B_ROW_MAJOR_KxN, GEMM_ERR_CUDA, GEMM_ERR_INVALID_ARG,  # noqa: F401
                   GEMM_ERR_TIMEOUT, GEMM_ERR_UNSUPPORTED, GEMM_OK, GemmError, check)
from .gemm import _stream

GEMM_TYPE_F32 = 0
GEMM_TYPE_BF16 = 1
GEMM_Q8_BLOCK = 32

GEMM_ACT_SILU = 0
GEMM_ACT_GELU = 1
GEMM_ACT_GELU_TANH = 2
GEMM_ACT_RELU = 3

_I64, _VP, _CI, _CF, _U64 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_uint64
_SIGNATURES = {
    "gemm_layernorm_forward": [_I64, _I64, _VP, _I64, _CI, _VP, _VP, _CI, _CF, _VP, _I64, _CI, _VP, _VP,
                               _VP, _I64, _VP, _I64, _VP],
    "gemm_layernorm_backward": [_I64, _I64, _VP, _I64, _CI, _VP, _I64, _VP, _I64, _VP, _CI, _VP, _VP,
                                _VP, _I64, _CI, _VP, _I64, _CI, _VP, _VP, _VP],
    "gemm_q8_save": [_I64, _I64, _VP, _I64, _CI, _VP, _I64, _VP, _I64, _VP],
    "gemm_q8_restore": [_I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _CI, _VP],
    "gemm_q8_weight_grad": [_I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _CI, _CI, _VP],
    "gemm_gated_forward": [_I64, _I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _CI, _CI, _VP, _I64, _VP, _I64, _VP,
                           _I64, _VP],
    "gemm_gated_backward": [_I64, _I64, _VP, _I64, _VP, _I64, _VP, _I64, _CI, _VP, _I64, _VP, _I64, _VP, _I64, _VP,
                            _I64, _VP],
    "gemm_gated_down_backward": [_I64, _I64, _I64, _VP, _I64, _VP, _I64, _CI, _VP, _I64, _VP, _I64, _CI, _VP, _I64,
                                 _VP, _I64, _VP, _I64, _VP, _I64, _VP],
    "gemm_dropout_forward": [_I64, _I64, _VP, _I64, _CI, _VP, _I64, _VP, _I64, _CI, _CF, _U64, _U64, _VP, _VP],
    "gemm_dropout_backward": [_I64, _I64, _VP, _I64, _CI, _VP, _I64, _CI, _CF, _U64, _U64, _VP, _VP],
}
_functions = {}


def library():
    """The loaded library with this header's functions typed."""
    lib = _gemm.library()
    for name, args in _SIGNATURES.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = _CI
        _functions[name] = f
    return lib


def _function(name):
    f = _functions.get(name)
    if f is None:
        library()
        f = _functions[name]
    return f


def _p(x):
    return x if x is None or isinstance(x, int) else x.data_ptr()


def gemm_layernorm_forward(rows, cols, x, ldx, x_type, gamma, beta, param_type, eps, y, ldy, y_type, mean, rstd,
                           q=None, ldq=0, e=None, lde=0, stream=None) -> int:
    """y = layer_norm(x) * gamma + beta by rows; the rows' mean and 1/std; with q and e, y's checkpoint too."""
    return _function("gemm_layernorm_forward")(rows, cols, _p(x), ldx, x_type, _p(gamma), _p(beta), param_type,
                                               eps, _p(y), ldy, y_type, _p(mean), _p(rstd), _p(q), ldq,
                                               _p(e), lde, _stream(stream))


def gemm_layernorm_backward(rows, cols, x, ldx, x_type, q, ldq, e, lde, gamma, param_type, mean, rstd, dy, lddy,
                            dy_type, dx, lddx, dx_type, dgamma, dbeta, stream=None) -> int:
    """dx, dgamma and dbeta of that layer norm from x, or from x's checkpoint (x None, q and e given)."""
    return _function("gemm_layernorm_backward")(rows, cols, _p(x), ldx, x_type, _p(q), ldq, _p(e), lde,
                                                _p(gamma), param_type, _p(mean), _p(rstd), _p(dy), lddy,
                                                dy_type, _p(dx), lddx, dx_type, _p(dgamma), _p(dbeta),
                                                _stream(stream))


def gemm_q8_save(rows, cols, x, ldx, x_type, q, ldq, e, lde, stream=None) -> int:
    """The 8-bit checkpoint (q, e) of x."""
    return _function("gemm_q8_save")(rows, cols, _p(x), ldx, x_type, _p(q), ldq, _p(e), lde, _stream(stream))


def gemm_q8_restore(rows, cols, q, ldq, e, lde, x, ldx, x_type, stream=None) -> int:
    """The values that a checkpoint stands for, into x."""
    return _function("gemm_q8_restore")(rows, cols, _p(q), ldq, _p(e), lde, _p(x), ldx, x_type, _stream(stream))


def gemm_q8_weight_grad(T, K, N, q, ldq, e, lde, dY, lddy, base, ldbase, dW, ldw, w_layout, w_type,
                        stream=None) -> int:
    """dW = base + X^T . dY, X (T x K) held as the checkpoint (q, e), dY (T x N) bf16; base None: zero."""
    return _function("gemm_q8_weight_grad")(T, K, N, _p(q), ldq, _p(e), lde, _p(dY), lddy, _p(base), ldbase,
                                            _p(dW), ldw, w_layout, w_type, _stream(stream))


def gemm_gated_forward(T, K, F, X, ldx, Wg, ldwg, Wu, ldwu, w_layout, activation, H, ldh, G=None, ldg=0, U=None,
                       ldu=0, stream=None) -> int:
    """H = act(X . Wg) * (X . Wu), bf16; with G and U, the two products too."""
    return _function("gemm_gated_forward")(T, K, F, _p(X), ldx, _p(Wg), ldwg, _p(Wu), ldwu, w_layout, activation,
                                           _p(H), ldh, _p(G), ldg, _p(U), ldu, _stream(stream))


def gemm_gated_backward(T, F, dH, lddh, G, ldg, U, ldu, activation, dG, lddg, dU, lddu, q=None, ldq=0, e=None, lde=0,
                        stream=None) -> int:
    """dG = dH * U * act'(G), dU = dH * act(G); with q and e, the checkpoint of act(G) * U."""
    return _function("gemm_gated_backward")(T, F, _p(dH), lddh, _p(G), ldg, _p(U), ldu, activation, _p(dG), lddg,
                                            _p(dU), lddu, _p(q), ldq, _p(e), lde, _stream(stream))


def gemm_gated_down_backward(T, N, F, dO, lddo, Wd, ldwd, w_layout, G, ldg, U, ldu, activation, dG, lddg, dU, lddu,
                             q=None, ldq=0, e=None, lde=0, stream=None) -> int:
    """The same from dO, with dH = dO . Wd^T taken in the same kernel."""
    return _function("gemm_gated_down_backward")(T, N, F, _p(dO), lddo, _p(Wd), ldwd, w_layout, _p(G), ldg, _p(U),
                                                 ldu, activation, _p(dG), lddg, _p(dU), lddu, _p(q), ldq, _p(e), lde,
                                                 _stream(stream))


def gemm_dropout_forward(rows, cols, x, ldx, x_type, residual, ldr, y, ldy, y_type, p, seed, step, step_device=None,
                         stream=None) -> int:
    """y = residual + keep * x / (1 - p); residual None: zero.  step_device: 8 bytes on the device added to step."""
    return _function("gemm_dropout_forward")(rows, cols, _p(x), ldx, x_type, _p(residual), ldr, _p(y), ldy, y_type, p,
                                             seed, step, _p(step_device), _stream(stream))


def gemm_dropout_backward(rows, cols, dy, lddy, dy_type, dx, lddx, dx_type, p, seed, step, step_device=None,
                          stream=None) -> int:
    """dx = keep * dy / (1 - p), keeping what the forward call of that seed and step kept."""
    return _function("gemm_dropout_backward")(rows, cols, _p(dy), lddy, dy_type, _p(dx), lddx, dx_type, p, seed, step,
                                              _p(step_device), _stream(stream))
