"""How the gated feed-forward and dropout calls run: captured and replayed, on
several streams at once, without scratch, the same from run to run, past 2^31
elements, and on sums that float32 holds exactly or that are hard on the tensor
core's additions."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from tests import gated_ref as A
from tests import layer_ref as R
from tests.test_gpu_gated import ACT, KN, NK, bf, check_backward, gate_inputs, weight
from tests.test_gpu_layer import Mat, _lib, done, within  # noqa: F401

pytestmark = pytest.mark.gpu

# few tokens; tiles in one round; a split tail; operands to be copied
SIZES = [(7, 200, 96), (300, 128, 264), (300, 4096, 520), (150, 333, 129)]


class Problem:
    """Both directions of a problem, and their calls on a stream."""

    def __init__(self, T, K, F, seed, layout=KN):
        rng = np.random.default_rng(seed)
        self.T, self.K, self.F, self.layout = T, K, F, layout
        self.x = bf(rng.normal(size=(T, K)))
        self.w = [bf(rng.normal(size=(K, F)) / K ** 0.5) for _ in range(3)]
        self.X, self.W = Mat(T, K, "bf16", fill=self.x), [weight(w, layout) for w in self.w]
        # Wd (F x K) as the transposed third weight: its layout is the other one
        self.back = NK if layout == KN else KN
        self.out = [Mat(T, F, "bf16") for _ in range(5)] + [Mat(T, F, "s8"), Mat(T, -(-F // 32), "u8")]

    def call(self, stream=None):
        H, Gm, U, dG, dU, Q, E = self.out
        T, K, F = self.T, self.K, self.F
        a = L.gemm_gated_forward(T, K, F, self.X.ptr, K, self.W[0].ptr, self.W[0].ld, self.W[1].ptr, self.W[1].ld,
                                 self.layout, ACT["silu"], H.ptr, F, Gm.ptr, F, U.ptr, F, stream=stream)
        b = L.gemm_gated_down_backward(T, K, F, self.X.ptr, K, self.W[2].ptr, self.W[2].ld, self.back, Gm.ptr, F, U.ptr,
                                       F, ACT["silu"], dG.ptr, F, dU.ptr, F, Q.ptr, F, E.ptr, E.ld, stream=stream)
        return a, b

    def results(self):
        return [m.view.clone() for m in self.out]

    def clear(self):
        for m in self.out:
            m.view.zero_()

    def check(self):
        H, Gm, U, dG, dU, Q, E = (m.host() for m in self.out)
        for got, (want, bound) in zip((H, Gm, U), A.forward(self.x, self.w[0], self.w[1], "silu")):
            within(got, want, bound)
        check_backward(*A.product(self.x, self.w[2]), Gm, U, "silu", [dG, dU], (Q, E))


@pytest.mark.parametrize("size", SIZES)
def test_captured_and_replayed(size):
    """A replay reads what lies in the inputs then, and gives the same bits as an
    eager call."""
    p = Problem(*size, 1)
    st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    assert p.call(st) == (0, 0)                            # the scratch grows outside the capture
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        status = p.call(st)
    assert status == (0, 0)
    p.x = bf(np.random.default_rng(9).normal(size=p.x.shape))
    p.X.view.copy_(torch.from_numpy(p.x))
    p.clear()
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    p.check()
    replayed = p.results()
    assert p.call() == (0, 0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(replayed, p.results()))


def test_captures_that_share_a_stream_s_scratch():
    """Two graphs captured on one stream, replayed in turn."""
    st = torch.cuda.Stream()
    problems = [Problem(*s, i) for i, s in enumerate((SIZES[2], SIZES[3]))]
    st.wait_stream(torch.cuda.current_stream())
    graphs = []
    for p in problems:
        assert p.call(st) == (0, 0)
    torch.cuda.synchronize()
    for p in problems:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=st):
            status = p.call(st)
        assert status == (0, 0)
        p.clear()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for i in (0, 1, 1, 0):
            graphs[i].replay()
    torch.cuda.synchronize()
    for p in problems:
        p.check()


def test_captures_without_scratch():
    """Aligned rows in whole rounds need no scratch; what needs some that its
    stream does not have is refused before anything is launched."""
    needs = {SIZES[0]: (0, 0), SIZES[2]: (G.GEMM_ERR_UNSUPPORTED,) * 2, SIZES[3]: (G.GEMM_ERR_UNSUPPORTED,) * 2}
    problems = {s: Problem(*s, 5) for s in needs}
    for p in problems.values():                            # kernels are loaded outside the capture
        assert p.call() == (0, 0)
    torch.cuda.synchronize()
    G.gemm_release_resources()                             # no stream has scratch
    for s, want in needs.items():
        st, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        before = G.gemm_launch_count()
        with torch.cuda.graph(graph, stream=st):
            status = problems[s].call(st)
        assert status == want and G.gemm_launch_count() - before == (2 if want == (0, 0) else 0)


def test_streams_at_once():
    problems = [Problem(*SIZES[i % 4], 20 + i, NK if i % 2 else KN) for i in range(8)]
    streams = [torch.cuda.Stream() for _ in problems]
    torch.cuda.synchronize()
    for _ in range(3):
        for p, st in zip(problems, streams):
            assert p.call(st) == (0, 0)
    torch.cuda.synchronize()
    assert G.gemm_device_status() == G.GEMM_OK
    for p in problems:
        p.check()


@pytest.mark.parametrize("size", SIZES + [(64, 2048, 512), (1100, 1024, 1504)])
def test_the_same_from_run_to_run(size):
    p = Problem(*size, 3)
    assert p.call() == (0, 0)
    first = p.results()
    for _ in range(3):
        p.clear()
        assert p.call() == (0, 0)
        assert all(torch.equal(a, b) for a, b in zip(first, p.results()))


@pytest.mark.parametrize("T,K,F", [(3, 512, 100), (64, 1024, 136), (200, 2048, 264), (520, 512, 777)])
@pytest.mark.parametrize("layout", [KN, NK])
def test_exact_sums(T, K, F, layout):
    """Small integers, whose sums float32 holds: G and U are the integers rounded
    to bf16, H with relu their exact product rounded."""
    rng = np.random.default_rng(T)
    x, wg, wu = (rng.integers(-3, 4, size=s).astype(np.float32) for s in ((T, K), (K, F), (K, F)))
    X, Wg, Wu = Mat(T, K, "bf16", fill=x), weight(wg, layout), weight(wu, layout)
    H, Gm, U = (Mat(T, F, "bf16") for _ in range(3))
    done(L.gemm_gated_forward(T, K, F, X.ptr, K, Wg.ptr, Wg.ld, Wu.ptr, Wu.ld, layout, ACT["relu"], H.ptr, F, Gm.ptr, F,
                              U.ptr, F))
    g, u = x.astype(np.float64) @ wg, x.astype(np.float64) @ wu
    assert np.abs(g).max() * np.abs(u).max() < 2 ** 24
    for m, want in ((Gm, g), (U, u), (H, np.maximum(g, 0) * u)):
        assert np.array_equal(m.host(), R.bf16_round(want.astype(np.float32)))


@pytest.mark.parametrize("T", [2, 130])
@pytest.mark.parametrize("K", [4096, 40000])
def test_one_large_and_many_small_products(T, K):
    """x = 1 and in each column of Wg one 1 among 0.98 * 2^-s, s from 20 to 31 in
    both signs: what the tensor core's additions cut stays within the contract."""
    F = 64
    rng = np.random.default_rng(K)
    j = np.arange(F)
    w = np.broadcast_to((63 / 64) * 2.0 ** -(20.0 + j % 12) * np.where(j // 12 % 2, -1, 1), (K, F)).copy()
    w[rng.integers(0, K, size=F), j] = np.where(j // 24 % 2, -1, 1)
    x, w = np.ones((T, K), np.float32), bf(w)
    X, W, one = Mat(T, K, "bf16", fill=x), Mat(K, F, "bf16", fill=w), Mat(K, F, "bf16", fill=bf(np.eye(K, F)))
    H, Gm, U = (Mat(T, F, "bf16") for _ in range(3))
    done(L.gemm_gated_forward(T, K, F, X.ptr, K, W.ptr, F, one.ptr, F, KN, ACT["silu"], H.ptr, F, Gm.ptr, F, U.ptr, F))
    g, c = w.astype(np.float64).sum(0), (K + 32) * 2.0 ** -24
    err = c * np.abs(w.astype(np.float64)).sum(0)
    within(Gm.host(), np.broadcast_to(g, (T, F)), err + (np.abs(g) + err) * 2.0 ** -8)
    assert (U.host() == 1).all()
    a = A.act(g, "silu")[0]
    err = 1.13 * err + c * np.abs(a) + 1.13 * c * err + A.ACT * np.abs(g)
    within(H.host(), np.broadcast_to(a, (T, F)), err + (np.abs(a) + err) * 2.0 ** -8)


@pytest.mark.parametrize("T,ld", [(5, 600_000_008), (5, 600_000_001), (200, 12_000_000), (200, 12_000_001)])
def test_rows_past_2_31_elements(T, ld):
    """Rows so far apart that their offsets pass 32 bits, in every T x F matrix at once."""
    K, F = 64, 40
    rng = np.random.default_rng(T)
    x, wg, wu, wd = (bf(rng.normal(size=s)) for s in ((T, K), (K, F), (K, F), (F, K)))
    big = torch.zeros(T * ld, dtype=torch.bfloat16, device="cuda")
    at = [big.data_ptr() + 2 * 64 * i for i in range(6)]   # matrices side by side in the rows
    view = [big.as_strided((T, F), (ld, 1), 64 * i) for i in range(6)]
    X, Wg, Wu, Wd = (Mat(*a.shape, "bf16", fill=a) for a in (x, wg, wu, wd))
    done(L.gemm_gated_forward(T, K, F, X.ptr, K, Wg.ptr, F, Wu.ptr, F, KN, ACT["gelu"], at[0], ld, at[1], ld, at[2], ld))
    H, Gm, U = (v.float().cpu().numpy() for v in view[:3])
    for got, (want, bound) in zip((H, Gm, U), A.forward(x, wg, wu, "gelu")):
        within(got, want, bound)
    d, ed = A.product(x, wd.T)
    for product in (True, False):
        Q, E = Mat(T, F, "s8"), Mat(T, 2, "u8")
        rest = (at[1], ld, at[2], ld, ACT["gelu"], at[4], ld, at[5], ld, Q.ptr, F, E.ptr, 2)
        if product:
            done(L.gemm_gated_down_backward(T, K, F, X.ptr, K, Wd.ptr, K, KN, *rest))
            dh, edh = d, ed
        else:
            dh, edh = bf(d), 0
            view[3].copy_(torch.from_numpy(dh))
            done(L.gemm_gated_backward(T, F, at[3], ld, *rest))
        check_backward(dh, edh, Gm, U, "gelu", [v.float().cpu().numpy() for v in view[4:]], (Q.host(), E.host()))
    done(L.gemm_dropout_forward(T, F, at[0], ld, 1, at[1], ld, at[3], ld, 1, 0.3, 4, 5))
    within(view[3].float().cpu().numpy(), *A.dropout(H, Gm, 0.3, 4, 5, "bf16"))


def test_many_elements():
    """More than 2^32 elements in one matrix, as one long pass: the last rows."""
    T, F = 140_000, 32_768                                  # 4.6e9 elements
    dh = torch.full((T, F), 0.5, dtype=torch.bfloat16, device="cuda")
    g, u = torch.full_like(dh, 1.0), torch.full_like(dh, 2.0)
    g[-1], u[-1, 5] = -1.0, 3.0
    done(L.gemm_gated_backward(T, F, dh, F, g, F, u, F, ACT["relu"], g, F, u, F))
    assert (g[T - 2] == 1).all() and (u[T - 2] == 0.5).all() and (g[-1] == 0).all() and (u[-1] == 0).all()
    assert (g[0] == 1).all() and (u[T // 2] == 0.5).all()
    done(L.gemm_dropout_backward(T, F, dh, F, 1, dh, F, 1, 0.5, 6, 7))
    # column groups and the row are the counter: the same as a small matrix of the last rows would draw
    groups = np.arange(F // 8, dtype=np.uint64)
    w = A.philox([groups, np.full(F // 8, T - 1, np.uint64), np.full(F // 8, 7, np.uint64), np.zeros(F // 8, np.uint64)],
                 (6, 0))
    n = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], 1).transpose(2, 0, 1).reshape(-1)
    assert np.array_equal(dh[-1].float().cpu().numpy(), np.where(n >= 32768, 1.0, 0.0))
