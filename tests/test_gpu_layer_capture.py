"""What a layer call needs of its stream's scratch when it is captured in a
CUDA graph: nothing where it uses none."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from tests import layer_ref as R
from tests.test_gpu_layer import TYPES, Mat, _lib, as_kind, vec, within  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(1, 4096), (4, 777), (4, 4096)])
def test_backward_of_few_rows_is_captured_on_a_stream_without_scratch(rows, cols):
    """Up to four rows are one block's, which writes dgamma and dbeta itself."""
    rng = np.random.default_rng(rows + cols)
    x, dy = (as_kind(rng.normal(size=(rows, cols)), "bf16") for _ in range(2))
    _, m, s = R.ln_forward(x, 1, 0, 1e-5)
    m, s = m.astype(np.float32), s.astype(np.float32)
    X, D, O = Mat(rows, cols, "bf16", fill=x), Mat(rows, cols, "bf16", fill=dy), Mat(rows, cols, "bf16")
    dg, db, mean, rstd = Mat(1, cols, "f32"), Mat(1, cols, "f32"), vec(m, "f32"), vec(s, "f32")

    def call(st):
        return L.gemm_layernorm_backward(rows, cols, X.ptr, cols, TYPES["bf16"], None, 0, None, 0, None, 0, mean, rstd,
                                         D.ptr, cols, TYPES["bf16"], O.ptr, cols, TYPES["bf16"], dg.ptr, db.ptr,
                                         stream=st)
    G.gemm_release_resources()                         # no stream has scratch
    assert call(torch.cuda.Stream()) == G.GEMM_OK      # the kernel is loaded outside the capture
    torch.cuda.synchronize()
    want = [a.view.clone() for a in (O, dg, db)]
    for a in (O, dg, db):
        a.view.zero_()
    torch.cuda.synchronize()
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        status = call(st)
    assert status == G.GEMM_OK, G.gemm_status_string(status)
    graph.replay()
    torch.cuda.synchronize()
    for a, w in zip((O, dg, db), want):
        assert torch.equal(a.view, w)
    ref, bound = R.ln_backward(x, m, s, 1, dy), R.ln_backward_bounds(x, m, s, 1, dy, "bf16")
    within(dg.host()[0], ref[1], bound[1])
