"""What the feed-forward block's dropout draws: blocks apart from one another,
passes and replays of a captured pass apart, the backward pass as its forward
pass."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import feed_forward_block as FB
from tests import gated_ref as A
from tests.test_gpu_layer import _lib  # noqa: F401

pytestmark = pytest.mark.gpu

T, K, F = 64, 64, 96


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def kept(x, y):
    """Where y = x + dropout(o) differs from x."""
    return (x != y).cpu().numpy()


def inputs(seed=1):
    gen = generator(seed)
    return [torch.randn((T, K), device="cuda", generator=gen) for _ in range(2)]


@pytest.mark.parametrize("shared", [True, False], ids=["one generator", "no generator"])
def test_blocks_made_alike_draw_apart(shared):
    """Layers of a stack: of two masks drawn apart at a half, positions agree by
    halves, within six standard deviations."""
    gen = generator(4) if shared else None
    x, _ = inputs()
    masks = [kept(x, FB.FeedForwardBlock(K, F, drop=0.5, generator=gen).forward(x)) for _ in range(3)]
    for i in range(3):
        agree = (masks[i] == masks[i - 1]).sum()
        assert abs(agree - T * K / 2) < 6 * (T * K / 4) ** 0.5
        assert abs(masks[i].sum() - T * K / 2) < 6 * (T * K / 4) ** 0.5


def test_a_generator_fixes_the_draws():
    x, _ = inputs()
    a, b = (FB.FeedForwardBlock(K, F, drop=0.5, generator=generator(6)) for _ in range(2))
    assert torch.equal(a.weight, b.weight) and torch.equal(a.forward(x), b.forward(x))


def test_a_seed_is_the_key():
    """... and leaves the weights as they are without one."""
    x, _ = inputs()
    a, b = (FB.FeedForwardBlock(K, F, drop=0.5, generator=generator(6), **kw) for kw in ({}, {"seed": 2 ** 63 + 5}))
    assert torch.equal(a.weight, b.weight) and torch.equal(a.down, b.down)
    assert np.array_equal(kept(x, b.forward(x)), A.keep(T, K, 0.5, 2 ** 63 + 5, 0))
