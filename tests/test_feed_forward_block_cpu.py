"""The gated feed-forward block refuses tensors that its calls would read past
or take for what they are not, before any call of the library (no GPU needed)."""
import pytest
import torch

from paper_2512_13282_gb300 import feed_forward_block as FB
from paper_2512_13282_gb300 import projection_block as PB

K, F, T = 64, 48, 4
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    """Every call of the library fails the test."""
    def called(*args, **kwargs):
        raise AssertionError("the library is called")
    for module in (FB.L, FB.G):
        for name in dir(module):
            if name.startswith("gemm_"):
                monkeypatch.setattr(module, name, called)


def block(held=None):
    b = object.__new__(FB.FeedForwardBlock)
    b.width, b.hidden, b.act, b.drop, b.eps, b.seed, b.step = K, F, "silu", 0.1, 1e-5, 0, 0
    b.gamma, b.beta = torch.ones(K), torch.zeros(K)
    b.weight, b.down = torch.zeros((K, 2 * F), dtype=BF16), torch.zeros((F, K), dtype=BF16)
    b._held = None
    if held is not None:
        b._held = (PB.Checkpoint(T, K, "cpu"), PB.Checkpoint(T, K, "cpu"), torch.zeros(T), torch.ones(T),
                   torch.zeros((T, 2 * F), dtype=BF16), held, 0)
    return b


@pytest.mark.parametrize("dy", [
    torch.zeros((T + 5, K), dtype=BF16), torch.zeros((T - 1, K), dtype=BF16), torch.zeros((T, K + 1), dtype=BF16),
    torch.zeros((T, K)), torch.zeros((T, K), dtype=torch.float16), torch.zeros((T, 2 * K), dtype=BF16)[:, ::2],
    torch.zeros((1, K), dtype=BF16).expand(T, K), torch.zeros((K, T), dtype=BF16).t(), torch.zeros(K, dtype=BF16),
    torch.zeros((T, K), dtype=BF16, device="meta")])
def test_backward_refuses(dy):
    b = block(BF16)
    with pytest.raises(ValueError):
        b.backward(dy)
    assert b._held is not None, "the activations stay held"


def test_a_backward_pass_that_fails_holds_nothing():
    """It may have written over G and U."""
    b = block(BF16)
    with pytest.raises(AssertionError, match="library"):
        b.backward(torch.zeros((T, K), dtype=BF16))
    with pytest.raises(RuntimeError):
        b.backward(torch.zeros((T, K), dtype=BF16))


def test_backward_without_a_forward_pass():
    with pytest.raises(RuntimeError):
        block().backward(torch.zeros((T, K), dtype=BF16))


@pytest.mark.parametrize("x", [
    torch.zeros((T, K + 8), dtype=BF16), torch.zeros((T, K - 8)), torch.zeros((T, K), dtype=torch.float16),
    torch.zeros((T, 2 * K))[:, ::2], torch.zeros((1, K)).expand(T, K), torch.zeros((K, T)).t(), torch.zeros(K),
    torch.zeros((T, K), device="meta")])
def test_forward_refuses(x):
    with pytest.raises(ValueError):
        block().forward(x)


@pytest.mark.parametrize("kw", [dict(act="tanh"), dict(drop=1.0), dict(drop=-0.1), dict(drop=float("nan"))])
def test_blocks_that_do_not_exist(kw):
    with pytest.raises(ValueError):
        FB.FeedForwardBlock(K, F, **kw)


def test_a_good_tensor_reaches_the_library():
    for x in (torch.zeros((T, 2 * K))[:, :K], torch.zeros((T, K), dtype=BF16)):
        with pytest.raises(AssertionError, match="library"):
            block().forward(x)
    with pytest.raises(AssertionError, match="library"):
        block(torch.float32).backward(torch.zeros((T, K + 8))[:, :K])
