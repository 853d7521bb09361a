"""The feed-forward block's backward pass: what it adds up, and in which
precision."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import feed_forward_block as FB
from tests import layer_ref as R
from tests.test_gpu_layer import _lib  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,F", [(200, 128, 192), (77, 130, 101)])
def test_dx_is_rounded_once(T, K, F, monkeypatch):
    """bf16: the layer norm's gradient and the residual's meet in float32, so
    that where they cancel the sum is off by its own rounding, not by theirs."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    b = FB.FeedForwardBlock(K, F, "silu", 0.1, gen, seed=7)
    x, dy = (torch.randn((T, K), device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    products, call = [], FB.G.gemm_bf16_f32acc_bf16

    def record(*args, **kw):
        status = call(*args, **kw)
        products.append(args[8].clone())
        return status
    monkeypatch.setattr(FB.G, "gemm_bf16_f32acc_bf16", record)
    b.forward(x)
    cx, _, mean, rstd, _, _, _ = b._held
    dx = b.backward(dy)
    at = (R.q8_values(cx.q.cpu().numpy(), cx.e.cpu().numpy()), mean.cpu().numpy(), rstd.cpu().numpy(),
          b.gamma.double().cpu().numpy(), products[-1].double().cpu().numpy())
    total = R.ln_backward(*at)[0] + dy.double().cpu().numpy()
    err = R.ln_backward_bounds(*at, "f32")[0]
    err = err + (np.abs(total) + err) * 2.0 ** -24          # the sum in float32
    assert dx.dtype == torch.bfloat16
    assert (np.abs(dx.double().cpu().numpy() - total) <= err + (np.abs(total) + err) * R.U_OUT["bf16"]).all()
