"""The gated feed-forward block (layer norm, gate, GEMMs, checkpoints, weight
gradients, dropout together) against 64-bit arithmetic, and its training loop."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import feed_forward_block as FB
from paper_2512_13282_gb300 import gemm as G
from tests import gated_ref as A
from tests import layer_ref as R
from tests.test_gpu_layer import _lib  # noqa: F401

pytestmark = pytest.mark.gpu


def host(t):
    return t.double().cpu().numpy()


def values(c):
    return R.q8_values(c.q.cpu().numpy(), c.e.cpu().numpy())


@pytest.mark.parametrize("T,K,F,act,drop,dtype", [(200, 128, 192, "silu", 0.1, torch.bfloat16),
                                                  (77, 130, 101, "gelu", 0.25, torch.float32),
                                                  (40, 64, 96, "relu", 0.0, torch.bfloat16),
                                                  (300, 96, 160, "gelu_tanh", 0.5, torch.float32),
                                                  (1, 72, 40, "silu", 0.1, torch.bfloat16),
                                                  (65, 33, 47, "silu", 0.1, torch.float32)])
def test_gradients(T, K, F, act, drop, dtype, monkeypatch):
    """Each gradient against the 64-bit formula on what its call read, so that a
    bound is that call's alone: what the block hands from call to call is taken
    from the calls themselves.  Two micro-batches accumulate."""
    kind = "f32" if dtype == torch.float32 else "bf16"
    gen = torch.Generator(device="cuda").manual_seed(3)
    b = FB.FeedForwardBlock(K, F, act, drop, gen, seed=77)
    b.gamma += 0.1 * torch.randn(K, device="cuda", generator=gen)
    seen = {}

    def record(module, name, *which):
        call = getattr(module, name)

        def wrapped(*args, **kw):
            status = call(*args, **kw)
            torch.cuda.synchronize()
            seen.setdefault(name, []).append([args[i].clone() if isinstance(args[i], torch.Tensor) else args[i]
                                              for i in which])
            return status
        monkeypatch.setattr(module, name, wrapped)
    record(FB.L, "gemm_layernorm_forward", 9)                # n
    record(FB.L, "gemm_gated_forward", 11)                   # H
    record(FB.L, "gemm_dropout_forward", 2)                  # o
    record(FB.L, "gemm_dropout_backward", 5)                 # do
    record(FB.L, "gemm_gated_down_backward", 13, 17, 19)     # [dG dU], q, e
    record(FB.G, "gemm_bf16_f32acc_bf16", 8)                 # o, dn
    want = {k: 0.0 for k in ("w", "d", "gamma", "beta")}
    bound = dict(want)
    W, Wd, g64 = host(b.weight), host(b.down), host(b.gamma)
    for step in range(2):
        seen.clear()
        x = torch.randn((T, K), device="cuda", generator=gen).to(dtype)
        dy = torch.randn((T, K), device="cuda", generator=gen).to(dtype)
        y = b.forward(x)
        cx, cn, mean, rstd, gu, _, _ = b._held
        n, h, o = (host(seen[k][0][0]) for k in ("gemm_layernorm_forward", "gemm_gated_forward", "gemm_dropout_forward"))
        GU = host(gu)
        ref = A.forward(n, W[:, :F], W[:, F:], act)
        for got, (r, e) in zip((h, GU[:, :F], GU[:, F:]), ref):
            assert (np.abs(got - r) <= e).all()
        r, e = A.product(h, Wd)
        assert (np.abs(o - r) <= e + (np.abs(r) + e) * 2.0 ** -8).all()
        r, e = A.dropout(o, host(x), drop, 77, step, kind)
        assert (np.abs(host(y) - r) <= e).all()

        dx = b.backward(dy)
        do = host(seen["gemm_dropout_backward"][0][0])
        r, e = A.dropout(host(dy), None, drop, 77, step, "bf16")
        assert (np.abs(do - r) <= e).all()
        dgu, q, ex = seen["gemm_gated_down_backward"][0]
        dGU = host(dgu)
        dg, du, hh = A.backward(*A.product(do, Wd.T), GU[:, :F], GU[:, F:], act)
        assert (np.abs(dGU[:, :F] - dg[0]) <= dg[1]).all() and (np.abs(dGU[:, F:] - du[0]) <= du[1]).all()
        assert A.held_ok(q.cpu().numpy(), ex.cpu().numpy(), *hh)
        hs = R.q8_values(q.cpu().numpy(), ex.cpu().numpy())
        for name, xs, ds in (("d", hs, do), ("w", values(cn), dGU)):
            r, mag = R.weight_grad(xs, ds, None, False)
            want[name], bound[name] = want[name] + r, bound[name] + 2.0 ** -20 * mag
        dn = host(seen["gemm_bf16_f32acc_bf16"][1][0])
        r, e = A.product(dGU, W.T)
        assert (np.abs(dn - r) <= e + (np.abs(r) + e) * 2.0 ** -8).all()
        m, s = mean.cpu().numpy(), rstd.cpu().numpy()
        lx, lg, lb = R.ln_backward(values(cx), m, s, g64, dn)
        ex, eg, eb = R.ln_backward_bounds(values(cx), m, s, g64, dn, kind)
        total = lx + host(dy)
        assert dx.dtype == dtype and (np.abs(host(dx) - total) <= ex + (np.abs(total) + ex) * R.U_OUT[kind]).all()
        for name, r, e in (("gamma", lg, eg), ("beta", lb, eb)):
            want[name], bound[name] = want[name] + r, bound[name] + e
    for name, got in (("w", b.dweight), ("d", b.ddown), ("gamma", b.dgamma), ("beta", b.dbeta)):
        # the second micro-batch is added with one more rounding of float32
        assert (np.abs(host(got) - want[name]) <= bound[name] + 2.0 ** -22 * np.abs(want[name])).all(), name


def test_gradients_against_differences():
    """The block's gradients along random directions against central
    differences of its own 64-bit form at the weights' step: the block's rounding
    to bf16 and 8 bits (a relative 2^-8 at each of a handful of places, of random
    signs over thousands of terms) leaves a directional derivative within 4 %."""
    T, K, F = 128, 64, 96
    gen = torch.Generator(device="cuda").manual_seed(5)
    b = FB.FeedForwardBlock(K, F, "silu", 0.25, gen, seed=9)
    x = torch.randn((T, K), device="cuda", generator=gen)
    dy = torch.randn((T, K), device="cuda", generator=gen)
    b.forward(x)
    dx = b.backward(dy)
    keep = A.keep(T, K, 0.25, 9, 0) * (65536 / (65536 - A.threshold(0.25)))

    def loss(x, w, d):
        n = R.ln_forward(x, 1, 0, b.eps)[0]
        gu = n @ w
        h = A.act(gu[:, :F], "silu")[0] * gu[:, F:]
        return float(((x + keep * (h @ d)) * host(dy)).sum())
    at = [host(x), host(b.weight), host(b.down)]
    for i, grad in enumerate((dx, b.dweight, b.ddown)):
        v = host(grad) / np.linalg.norm(host(grad))       # along the gradient itself, where it is largest
        lo, hi = ([a - s * 1e-4 * v if j == i else a for j, a in enumerate(at)] for s in (1, -1))
        slope = (loss(*hi) - loss(*lo)) / 2e-4
        assert abs(slope - np.linalg.norm(host(grad))) < 0.04 * slope


def test_training_runs():
    launches = G.gemm_launch_count()
    losses = FB.train(300, 128, 160, 4, drop=0.1, report=lambda line: None)
    assert G.gemm_launch_count() > launches and np.isfinite(losses).all()


def test_steps_draw_apart_and_the_backward_pass_draws_the_same():
    b = FB.FeedForwardBlock(64, 64, "relu", 0.5, seed=3)
    x = torch.randn((16, 64), device="cuda")
    kept = []
    for step in range(2):
        y = b.forward(x)
        dropped = y == x
        ones = torch.ones_like(x)
        b.ddown.zero_()
        b.backward(ones)
        kept.append(~dropped.cpu().numpy())
        k = A.keep(16, 64, 0.5, 3, step)
        assert (dropped.cpu().numpy() | k).all() and not (kept[-1] & ~k).any()
    assert (kept[0] != kept[1]).any()


def test_no_tokens():
    b = FB.FeedForwardBlock(64, 96, drop=0.1)
    x = torch.empty((0, 64), device="cuda")
    assert b.forward(x).shape == (0, 64) and b.backward(x).shape == (0, 64)
    assert not any(g.any() for g in (b.dgamma, b.dbeta, b.dweight, b.ddown))


def test_a_captured_pass():
    """Both passes in a graph, with a block that runs eagerly beside it: the
    replay gives what the eager passes give, of the inputs it finds then."""
    T, K, F = 200, 64, 96
    gen = torch.Generator(device="cuda").manual_seed(8)
    b = FB.FeedForwardBlock(K, F, "silu", 0.25, gen, seed=9)
    x, dy = (torch.randn((T, K), device="cuda", generator=gen) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.forward(x)
        b.backward(dy)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.step = 5
            b.zero_grad()
            y = b.forward(x)
            dx = b.backward(dy)
        for _ in range(2):
            x.copy_(torch.randn((T, K), device="cuda", generator=gen))
            graph.replay()
            got = [t.clone() for t in (y, dx, b.dweight, b.ddown, b.dgamma, b.dbeta)]
            b.step = 5
            b.zero_grad()
            want = [b.forward(x), b.backward(dy), b.dweight, b.ddown, b.dgamma, b.dbeta]
            assert all(torch.equal(g, w) for g, w in zip(got, want))
    torch.cuda.current_stream().wait_stream(side)
