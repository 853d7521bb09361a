"""The blocks' passes on two streams: what the forward pass leaves is not handed
out to the forward pass's stream while the backward pass of another one has yet
to read it."""
import pytest
import torch

from paper_2512_13282_gb300 import feed_forward_block as FB
from paper_2512_13282_gb300 import projection_block as PB
from tests.test_gpu_layer import _lib  # noqa: F401

pytestmark = pytest.mark.gpu

T, K, F = 512, 256, 1024


def feed_forward():
    gen = torch.Generator(device="cuda").manual_seed(2)
    b = FB.FeedForwardBlock(K, F, "silu", 0.25, gen, seed=5)
    return b, torch.randn((T, K), device="cuda", generator=gen), lambda: [b.dweight, b.ddown, b.dgamma]


def projection():
    gen = torch.Generator(device="cuda").manual_seed(2)
    b = PB.ProjectionBlock(K, F, gen)
    return b, torch.randn((T, F), device="cuda", generator=gen).to(torch.bfloat16), lambda: [b.dweight, b.dgamma, b.dbeta]


def tensors(held):
    for h in held:
        if isinstance(h, PB.Checkpoint):
            yield from (h.q, h.e)
        elif isinstance(h, torch.Tensor):
            yield h


@pytest.mark.parametrize("make", [feed_forward, projection])
def test_a_backward_pass_on_another_stream(make):
    results = []
    for apart in (False, True):
        b, dy, grads = make()
        x = torch.randn((T, K), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
        one = torch.cuda.Stream()
        two = torch.cuda.Stream() if apart else one
        one.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(one):
            b.forward(x)
            held = list(tensors(b._held))
            places, shapes = {t.data_ptr() for t in held}, [(t.shape, t.dtype) for t in held]
            del held
            # as much again, free on this stream: what follows asks the driver for none
            spare = [torch.empty(s, dtype=d, device="cuda") for s, d in shapes]
            del spare
        torch.cuda.synchronize()
        with torch.cuda.stream(two):
            if apart:
                torch.cuda._sleep(200_000_000)         # 0.1 s and no more
            dx = b.backward(dy)
        if apart:
            assert not two.query(), "the backward pass has yet to run"
            with torch.cuda.stream(one):
                new = [torch.full(s, 77, dtype=d, device="cuda") for s, d in shapes]
            assert not places & {t.data_ptr() for t in new}
        torch.cuda.synchronize()
        results.append([dx.clone()] + [g.clone() for g in grads()])
    assert all(torch.equal(a, b) for a, b in zip(*results))
