"""The projection block (layer norm, GEMMs, checkpoints, weight gradient
together) against 64-bit arithmetic, and its training loop."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from paper_2512_13282_gb300 import projection_block as PB
from tests import layer_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2512_13282_gb300 import build
    build.build()
    L.library()


@pytest.mark.parametrize("T,K,N,dtype", [(200, 256, 320, torch.bfloat16), (77, 333, 129, torch.float32)])
def test_gradients(T, K, N, dtype):
    """Each gradient against the 64-bit formula on what its call read: the
    weight gradient on y's checkpoint and do, dx, dgamma and dbeta on x's
    checkpoint and the bf16 dy = do . W^T, which is itself within the GEMM's
    bound.  Two micro-batches accumulate."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    b = PB.ProjectionBlock(K, N, gen)
    b.gamma += 0.1 * torch.randn(K, device="cuda", generator=gen)
    dw = mag_w = dg = db = 0.0
    dg_bound = db_bound = 0.0
    for _ in range(2):
        x = torch.randn((T, K), device="cuda", generator=gen).to(dtype)
        do = torch.randn((T, N), device="cuda", generator=gen).to(torch.bfloat16)
        o = b.forward(x)
        cx, cy, mean, rstd, _ = b._held
        xs, ys = (R.q8_values(c.q.cpu().numpy(), c.e.cpu().numpy()) for c in (cx, cy))
        # the checkpoints are those of x and of the y that the GEMM read
        q, e = R.q8_save(x.float().cpu().numpy())
        assert np.array_equal(cx.q.cpu().numpy(), q) and np.array_equal(cx.e.cpu().numpy(), e)
        g64, W = b.gamma.double().cpu().numpy(), b.weight.double().cpu().numpy()
        y64, _, _ = R.ln_forward(x.float().cpu().numpy(), g64, b.beta.double().cpu().numpy(), b.eps)
        # o: bf16 y (half a unit, 2^-8 relative, plus its float32 error) through W, then rounded
        y_err = R.ln_forward_bounds(x.float().cpu().numpy(), g64, b.beta.double().cpu().numpy(), b.eps, "bf16")[0]
        ref = y64 @ W
        o_err = y_err @ np.abs(W) + 2.0 ** -20 * (np.abs(y64) + y_err) @ np.abs(W)
        assert (np.abs(o.double().cpu().numpy() - ref) <= o_err + 2.0 ** -8 * (np.abs(ref) + o_err)).all()
        dx = b.backward(do)
        d64 = do.double().cpu().numpy()
        dy = d64 @ W.T
        dy_err = 2.0 ** -8 * np.abs(dy) * 1.01 + 2.0 ** -20 * np.abs(d64) @ np.abs(W.T)
        m, s = mean.cpu().numpy(), rstd.cpu().numpy()
        want = R.ln_backward(xs, m, s, g64, dy)
        bound = R.ln_backward_bounds(xs, m, s, g64, dy, "f32" if dtype == torch.float32 else "bf16")
        xh = np.abs((xs - m[:, None].astype(np.float64)) * s[:, None].astype(np.float64))
        g_err = dy_err * np.abs(g64)
        spread = s[:, None] * (g_err + g_err.mean(1, keepdims=True) + xh * (g_err * xh).mean(1, keepdims=True))
        got = dx.double().cpu().numpy()
        assert dx.dtype == dtype and (np.abs(got - want[0]) <= bound[0] + 1.01 * spread).all()
        dg, db = dg + want[1], db + want[2]
        dg_bound = dg_bound + bound[1] + (dy_err * xh).sum(0) + 2.0 ** -23 * np.abs(dg)
        db_bound = db_bound + bound[2] + dy_err.sum(0) + 2.0 ** -23 * np.abs(db)
        r, mag = R.weight_grad(ys, d64, None, False)
        dw, mag_w = dw + r, mag_w + mag
    assert (np.abs(b.dgamma.double().cpu().numpy() - dg) <= dg_bound).all()
    assert (np.abs(b.dbeta.double().cpu().numpy() - db) <= db_bound).all()
    got = b.dweight.double().cpu().numpy()
    assert (np.abs(got - dw) <= 2 * R.weight_grad_bound(dw, mag_w, "f32")).all()


def test_training_lowers_the_loss():
    launches = G.gemm_launch_count()
    losses = PB.train(512, 256, 192, 25, report=lambda line: None)
    assert G.gemm_launch_count() > launches
    assert losses[-1] < 0.5 * losses[0] and all(np.isfinite(losses))
