"""The layer operators' checks at sizes where a block takes several wide rows,
or a thread block several tiles whose base is fetched across tiles."""
import pytest

from tests import test_gpu_layer as checks
from tests.test_gpu_layer import _lib  # noqa: F401

pytestmark = pytest.mark.gpu

WIDE = [(640, 4104), (500, 5120), (420, 5690), (330, 6200), (480, 4096), (320, 8192), (310, 12281)]


@pytest.mark.parametrize("rows,cols", WIDE)
@pytest.mark.parametrize("xt,yt,pt", [("bf16", "bf16", "f32"), ("f32", "f32", "bf16")])
def test_layernorm_forward_of_wide_rows(rows, cols, xt, yt, pt):
    checks.test_layernorm_forward(rows, cols, xt, yt, pt)


@pytest.mark.parametrize("rows,cols", WIDE)
@pytest.mark.parametrize("xt,gt,ot", [("bf16", "bf16", "bf16"), ("q8", "bf16", "f32")])
def test_layernorm_backward_of_wide_rows(rows, cols, xt, gt, ot):
    checks.test_layernorm_backward_of_many_rows(rows, cols, xt, gt, ot)


@pytest.mark.parametrize("rows,cols", [(700, 1501), (40, 10471), (3000, 33)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_checkpoint_of_many_unaligned_rows(rows, cols, kind):
    checks.test_checkpoint(rows, cols, kind)


@pytest.mark.parametrize("T,K,N", [(100, 2500, 2000), (1, 2048, 2560), (512, 2304, 2056), (600, 3000, 2504),
                                   (768, 1000, 4096)])
@pytest.mark.parametrize("wt", ["f32", "bf16"])
@pytest.mark.parametrize("nk", [False, True])
def test_weight_grad_of_many_tiles(T, K, N, wt, nk):
    checks.test_weight_grad(T, K, N, wt, nk)
