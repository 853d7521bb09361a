"""The weight gradient on inputs that are hard on its tensor-core chains: one
large product and many that a float32 sum beside it cannot hold."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import layer as L
from tests import layer_ref as R
from tests.test_gpu_layer import TYPES, Mat, _lib, as_kind, done, within  # noqa: F401

pytestmark = pytest.mark.gpu


def test_bf16_weight_grad_of_very_many_tokens():
    """X = 1, and in dY one token in 2^18 is 1 and the others 0.98 * 2^-25.  A
    chain of tensor-core additions that has reached 1 takes up none of the
    latter: over all of a part's tokens (the reduction is split 16 ways at most)
    that would lose 2^18 * 0.98 * 2^-25 = 0.8 % of it, twice what bf16's last
    rounding may be off.  Chains of a bounded length lose their own part only."""
    T, n, gap = 1 << 22, 64, 1 << 18
    q = torch.full((T, n), 64, dtype=torch.int8, device="cuda")
    e = torch.full((T, n // 32), 121, dtype=torch.uint8, device="cuda")       # 64 * 2^-6
    small = 63 * 2.0 ** -31
    dy = torch.full((T, n), small, dtype=torch.bfloat16, device="cuda")
    dy[::gap] = 1
    dy[:, 1::2] *= -1
    w = torch.empty((n, n), dtype=torch.bfloat16, device="cuda")
    done(L.gemm_q8_weight_grad(T, n, n, q, n, e, n // 32, dy, n, None, 0, w, n, L.GEMM_B_ROW_MAJOR_KxN,
                               L.GEMM_TYPE_BF16))
    ref = (T // gap + (T - T // gap) * small) * np.where(np.arange(n) % 2, -1.0, 1.0)
    within(w.float().cpu().numpy(), np.broadcast_to(ref, (n, n)), 2.0 ** -8 * np.abs(ref) * (1 + 2.0 ** -7))


@pytest.mark.parametrize("T,K,N", [(8193, 130, 70), (9000, 320, 300), (16500, 64, 257), (12345, 600, 1100)])
@pytest.mark.parametrize("nk", [False, True])
def test_bf16_weight_grad_of_many_tokens(T, K, N, nk):
    """Reductions past one chain, with and without a base, aligned and not."""
    rng = np.random.default_rng(T)
    shape = (N, K) if nk else (K, N)
    for pad, off, with_base in ((0, 0, False), (8, 0, True), (3, 1, True)):
        q = rng.integers(-127, 128, size=(T, K)).astype(np.int8)
        e = rng.integers(118, 122, size=(T, -(-K // 32))).astype(np.uint8)
        dy = as_kind(rng.normal(size=(T, N)), "bf16")
        base = as_kind(10 * rng.normal(size=shape), "bf16") if with_base else None
        Q, E, D = Mat(T, K, "s8", pad, off, q), Mat(T, e.shape[1], "u8", pad, off, e), Mat(T, N, "bf16", pad, off, dy)
        W, B = Mat(*shape, "bf16", pad, off), Mat(*shape, "bf16", pad, off, base) if with_base else None
        done(L.gemm_q8_weight_grad(T, K, N, Q.ptr, Q.ld, E.ptr, E.ld, D.ptr, D.ld, B.ptr if B else None,
                                   B.ld if B else 0, W.ptr, W.ld,
                                   L.GEMM_B_COL_MAJOR_NxK if nk else L.GEMM_B_ROW_MAJOR_KxN, TYPES["bf16"]))
        ref, mag = R.weight_grad(R.q8_values(q, e), dy, base, nk)
        within(W.host(), ref, R.weight_grad_bound(ref, mag, "bf16"))
        assert W.guarded()
