"""The step that a feed-forward block's dropout draws with is a 64-bit number
(no GPU needed)."""
import pytest

from paper_2512_13282_gb300 import feed_forward_block as FB


@pytest.mark.parametrize("value", [0, 5, 2 ** 63 - 1, 2 ** 63, 2 ** 64 - 1])
def test_the_step_holds_64_bits(value):
    b = object.__new__(FB.FeedForwardBlock)
    b.step = value
    assert b.step == value
    b._start += 1                                      # as a forward pass does
    assert b.step == (value + 1) % 2 ** 64
    b.step = value - 2 ** 64                           # modulo 2^64
    assert b.step == value
