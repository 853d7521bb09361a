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


def test_replays_draw_anew():
    """Each replay of a captured step draws with the next step, in both of its
    passes, and so do eager passes between them and another graph's replays: what
    a block beside it gives whose step is set to that."""
    x, dy = inputs()
    b, other = (FB.FeedForwardBlock(K, F, "silu", 0.5, generator(8), seed=9) for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def passes(block):
        block.zero_grad()
        return [block.forward(x), block.backward(dy), block.dweight, block.ddown]
    with torch.cuda.stream(side):
        passes(b)                                      # step 0
        side.synchronize()
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = passes(b)
            graphs.append((graph, out))

        def check(which, step):
            if which is None:
                got = passes(b)
            else:
                graphs[which][0].replay()
                got = graphs[which][1]
            got = [t.clone() for t in got]
            other.step = step
            want = passes(other)
            assert np.array_equal(kept(x, got[0]), A.keep(T, K, 0.5, 9, step))
            assert all(torch.equal(g, w) for g, w in zip(got, want))
        for step, which in enumerate((0, 0, None, 1, 0, None, None, 1), 1):
            check(which, step)
        assert b.step == 9
        for step in (100, 2 ** 64 - 1):
            b.step = step                              # past it, modulo 2^64
            assert b.step == step
            check(1, step)
            check(None, (step + 1) % 2 ** 64)
            check(0, (step + 2) % 2 ** 64)
    torch.cuda.current_stream().wait_stream(side)


def test_a_step_set_within_a_capture_is_set_by_its_replays():
    x, _ = inputs()
    b = FB.FeedForwardBlock(K, F, "silu", 0.5, generator(8), seed=9)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.forward(x)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            b.step = 30
            y = b.forward(x)
        for _ in range(3):
            graph.replay()
            assert np.array_equal(kept(x, y), A.keep(T, K, 0.5, 9, 30))
        assert b.step == 31
        assert np.array_equal(kept(x, b.forward(x)), A.keep(T, K, 0.5, 9, 31))
    torch.cuda.current_stream().wait_stream(side)


def test_the_step_is_read_and_set():
    x, _ = inputs()
    b = FB.FeedForwardBlock(K, F, "silu", 0.5, generator(8), seed=3)
    assert b.step == 0
    b.forward(x)
    assert b.step == 1
    for step in (7, 2 ** 63 + 1, 2 ** 64 - 1):
        b.step = step
        assert b.step == step
        assert np.array_equal(kept(x, b.forward(x)), A.keep(T, K, 0.5, 3, step))
    assert b.step == 0                                 # modulo 2^64


def test_the_backward_pass_draws_as_its_forward_pass(monkeypatch):
    """The gradient that goes into the down projection is zero where the forward
    pass dropped and doubled elsewhere, whatever the step is set to in between."""
    x, _ = inputs()
    b = FB.FeedForwardBlock(K, F, "silu", 0.5, generator(8), seed=3)
    seen, call = [], FB.L.gemm_dropout_backward

    def record(*args, **kw):
        status = call(*args, **kw)
        seen.append(args[5].clone())
        return status
    monkeypatch.setattr(FB.L, "gemm_dropout_backward", record)
    for step in (0, 1, 40):
        if step == 40:
            b.step = 40
        y = b.forward(x)
        b.step = step + 1
        b.backward(torch.ones_like(x))
        mask = A.keep(T, K, 0.5, 3, step)
        assert np.array_equal(kept(x, y), mask)
        assert np.array_equal(seen[-1].float().cpu().numpy(), 2 * mask.astype(np.float32))
