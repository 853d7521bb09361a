"""The bf16 GEMM's accuracy contract for all inputs, on sums that are hard on the
tensor core's additions: large products that cancel among many small ones, whose
sum is what is left."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import gemm as G
from tests.test_gpu_layer import _lib, done  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [512, 1024, 4096, 40000])
@pytest.mark.parametrize("M", [1, 2, 16, 130, 300])
@pytest.mark.parametrize("layout", [G.GEMM_B_ROW_MAJOR_KxN, G.GEMM_B_COL_MAJOR_NxK], ids=["KxN", "NxK"])
def test_large_products_that_cancel(M, K, layout):
    """A of ones; a column of B has 1 first and -1 last, or the other way round,
    and in between 0.98 * 2^-s of one sign, s from 20 to 31."""
    N = 64
    j = np.arange(N)
    b = np.broadcast_to((63 / 64) * 2.0 ** -(20.0 + j % 12) * np.where(j // 12 % 2, -1, 1), (K, N)).copy()
    b[0] = np.where(j // 24 % 2, -1, 1)
    b[K - 1] = -b[0]
    a = torch.ones((M, K), dtype=torch.bfloat16, device="cuda")
    B = torch.from_numpy(b).to(torch.bfloat16).cuda()
    assert np.array_equal(B.double().cpu().numpy(), b)
    if layout == G.GEMM_B_COL_MAJOR_NxK:
        B = B.t().contiguous()
    C = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    done(G.gemm_bf16_f32acc_bf16(M, N, K, a, K, B, B.stride(0), layout, C, N))
    ref, err = b.sum(0), (K + 32) * 2.0 ** -24 * np.abs(b).sum(0)
    assert (np.abs(C.double().cpu().numpy() - ref) <= 2.0 ** -8 * (np.abs(ref) + err) + err).all()
