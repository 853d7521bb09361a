"""The projection block refuses tensors that its calls would read past or take
for what they are not, before any call of the library (no GPU needed)."""
import pytest
import torch

from paper_2512_13282_gb300 import projection_block as PB

K, N, T = 64, 48, 4
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    """Every call of the library fails the test."""
    def called(*args, **kwargs):
        raise AssertionError("the library is called")
    for module in (PB.L, PB.G):
        for name in dir(module):
            if name.startswith("gemm_"):
                monkeypatch.setattr(module, name, called)


def block(held=True):
    b = object.__new__(PB.ProjectionBlock)
    b.width, b.out, b.eps = K, N, 1e-5
    b.gamma, b.beta = torch.ones(K), torch.zeros(K)
    b.weight = torch.zeros((K, N), dtype=BF16)
    b.dgamma, b.dbeta, b.dweight = torch.zeros(K), torch.zeros(K), torch.zeros((K, N))
    b._held = None
    if held:
        b._held = (PB.Checkpoint(T, K, "cpu"), PB.Checkpoint(T, K, "cpu"), torch.zeros(T), torch.ones(T), BF16)
    return b


@pytest.mark.parametrize("do", [
    torch.zeros((T + 5, N), dtype=BF16), torch.zeros((T - 1, N), dtype=BF16), torch.zeros((T, N + 1), dtype=BF16),
    torch.zeros((T, N)), torch.zeros((T, N), dtype=torch.float16), torch.zeros((T, 2 * N), dtype=BF16)[:, ::2],
    torch.zeros((1, N), dtype=BF16).expand(T, N), torch.zeros((N, T), dtype=BF16).t(), torch.zeros(N, dtype=BF16),
    torch.zeros((T, N), dtype=BF16, device="meta")])
def test_backward_refuses(do):
    b = block()
    with pytest.raises(ValueError):
        b.backward(do)
    assert b._held is not None, "the activations stay held"


def test_backward_without_a_forward_pass():
    with pytest.raises(RuntimeError):
        block(held=False).backward(torch.zeros((T, N), dtype=BF16))


BAD_X = [torch.zeros((T, K + 8), dtype=BF16), torch.zeros((T, K - 8)), torch.zeros((T, K), dtype=torch.float16),
         torch.zeros((T, K), dtype=torch.int16), torch.zeros((T, 2 * K))[:, ::2], torch.zeros((1, K)).expand(T, K),
         torch.zeros((K, T)).t(), torch.zeros(K), torch.zeros((T, K), device="meta")]


@pytest.mark.parametrize("x", BAD_X)
def test_forward_refuses(x):
    with pytest.raises(ValueError):
        block(held=False).forward(x)


@pytest.mark.parametrize("x", BAD_X + [torch.zeros((T + 1, K))])
def test_checkpoint_refuses(x):
    with pytest.raises(ValueError):
        PB.Checkpoint(T, K, "cpu").save(x)


def test_restore_refuses_other_types():
    with pytest.raises(ValueError):
        PB.Checkpoint(T, K, "cpu").restore(torch.float16)


def test_a_good_tensor_reaches_the_library():
    """The checks let through what they should: rows of a wider buffer, one row
    of any stride."""
    for x in (torch.zeros((T, 2 * K))[:, :K], torch.zeros((T, K), dtype=BF16)):
        with pytest.raises(AssertionError, match="library"):
            PB.Checkpoint(T, K, "cpu").save(x)
    with pytest.raises(AssertionError, match="library"):
        PB.Checkpoint(1, K, "cpu").save(torch.zeros((1, K)).expand(1, K))
    with pytest.raises(AssertionError, match="library"):
        block().backward(torch.zeros((T, N + 8), dtype=BF16)[:, :N])
