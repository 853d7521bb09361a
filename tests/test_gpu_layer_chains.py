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


def contract(T, ref, total, w_type):
    """The header's bound: chains of L tokens, of which 16 at a time cut 17 terms
    to 2^-25 of the largest and their sum to a float32, 10.5 * 2^-24 of the
    magnitudes' sum at most; a rounding for each chain, split part and base."""
    chain = {"f32": 512, "bf16": 8192}[w_type]
    err = (min(T, chain) + T / chain + 32) * 2.0 ** -24 * total
    return err + (np.abs(ref) + err) * R.U_OUT[w_type]


@pytest.mark.parametrize("T,K,N", [(16, 64, 64), (48, 96, 130), (512, 64, 96), (513, 32, 200), (512, 2048, 1100),
                                   (2000, 160, 480), (8192, 64, 64), (20000, 64, 64)])
@pytest.mark.parametrize("wt", ["f32", "bf16"])
@pytest.mark.parametrize("with_base", [False, True])
def test_weight_grad_of_one_large_and_many_small_products(T, K, N, wt, with_base):
    """X = 1; each column of dY has 1 at some token and 0.98 * 2^-s elsewhere, s
    from 20 to 31, in all four pairs of signs: what the additions cut adds up."""
    rng = np.random.default_rng(T + N)
    j = np.arange(N)
    dy = np.broadcast_to((63 / 64) * 2.0 ** -(20.0 + j % 12) * np.where(j // 12 % 2, -1, 1), (T, N)).copy()
    dy[rng.integers(0, T, size=N), j] = np.where(j // 24 % 2, -1, 1)
    if T > 100:
        dy[0, : N // 2] = 1                         # in the first step of the chain
    base = as_kind(rng.normal(size=(K, N)), wt) if with_base else np.zeros((K, N), np.float32)
    Q, E = Mat(T, K, "s8", fill=np.full((T, K), 64, np.int8)), Mat(T, K // 32, "u8", fill=np.full((T, K // 32), 121))
    D, W, B = Mat(T, N, "bf16", fill=dy), Mat(K, N, wt), Mat(K, N, wt, fill=base)
    done(L.gemm_q8_weight_grad(T, K, N, Q.ptr, K, E.ptr, K // 32, D.ptr, N, B.ptr if with_base else None, N, W.ptr, N,
                               L.GEMM_B_ROW_MAJOR_KxN, TYPES[wt]))
    ref, total = dy.sum(0) + base.astype(np.float64), np.abs(dy).sum(0) + np.abs(base.astype(np.float64))
    within(W.host(), ref, contract(T, ref, total, wt))
