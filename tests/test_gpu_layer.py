"""The layer operators on the GPU against their definitions in 64 bits
(tests/layer_ref.py), within bounds derived from the float32 operations they
take; checkpoints bit for bit.  Every output lies in a guarded buffer: nothing
outside its matrix may change."""
import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from tests import layer_ref as R

pytestmark = pytest.mark.gpu

TYPES = {"f32": L.GEMM_TYPE_F32, "bf16": L.GEMM_TYPE_BF16}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "s8": torch.int8, "u8": torch.uint8}
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2512_13282_gb300 import build
    build.build()
    L.library()


class Mat:
    """A rows x cols device matrix of pitch cols + pad, `off` elements into a
    buffer filled with a guard byte pattern."""

    def __init__(self, rows, cols, kind, pad=0, off=0, fill=None):
        self.rows, self.cols, self.ld, self.kind = rows, cols, cols + pad, kind
        dt = TORCH[kind]
        size = off + rows * self.ld + 8
        raw = torch.full((size * torch.empty(0, dtype=dt).element_size(),), 0x5A, dtype=torch.uint8, device="cuda")
        self.buf = raw.view(dt)
        self.off = off
        self.view = self.buf[off:off + rows * self.ld].view(rows, self.ld)[:, :cols]
        self.ptr = self.buf.data_ptr() + off * self.buf.element_size()
        if fill is not None:
            self.view.copy_(torch.from_numpy(np.ascontiguousarray(fill)))

    def host(self):
        v = self.view
        return (v.float() if v.is_floating_point() else v).cpu().numpy()

    def guarded(self):
        b = self.buf.view(torch.uint8).cpu().numpy().reshape(-1, self.buf.element_size())
        keep = np.ones(len(b), bool)
        body = keep[self.off:self.off + self.rows * self.ld].reshape(self.rows, self.ld)
        body[:, :self.cols] = False
        return (b[keep] == 0x5A).all()


def vec(a, kind):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(TORCH[kind])


def done(status):
    assert status == G.GEMM_OK, G.gemm_status_string(status)
    torch.cuda.synchronize()
    assert G.gemm_device_status() == G.GEMM_OK


def activations(rng, rows, cols, kind):
    x = rng.normal(size=(rows, cols)) * np.exp(0.5 * rng.normal(size=cols)) + 0.3 * rng.normal(size=cols)
    if cols > 4:
        x[:, cols // 3] *= 20                       # an outlier channel
    if rows > 2:
        x[rows // 2] = 3.0                          # a constant row: variance 0
        x[rows - 1] += 100.0                        # a mean far above the deviations
    return as_kind(x, kind)


def as_kind(x, kind):
    x = np.asarray(x, np.float32)
    return R.bf16_round(x) if kind == "bf16" else x


def within(got, want, bound):
    bad = ~(np.abs(got.astype(np.float64) - want) <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} values off, worst {np.nanmax(np.abs(got - want) / bound)} bounds"


# every width class: one value, below and across a warp, a vector, a block of
# 32; the repository's own widths; past what a block keeps in registers
SHAPES = [(1, 1), (1, 4096), (2, 7), (3, 31), (5, 32), (4, 33), (9, 64), (40, 96), (33, 777), (300, 1000), (7, 1500),
          (64, 2048), (1024, 512), (257, 4096), (20, 8192), (5, 8200), (6, 12288), (3, 16384), (2, 16392), (2, 40000)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("xt,yt,pt", [("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("f32", "bf16", "f32"),
                                      ("f32", "f32", "bf16")])
def test_layernorm_forward(rows, cols, xt, yt, pt):
    rng = np.random.default_rng(rows * 1000 + cols)
    for pad, off in ((0, 0), (8, 0), (3, 1)):
        x = activations(rng, rows, cols, xt)
        gamma, beta = as_kind(1 + 0.2 * rng.normal(size=cols), pt), as_kind(0.2 * rng.normal(size=cols), pt)
        X, Y = Mat(rows, cols, xt, pad, off, x), Mat(rows, cols, yt, pad, off)
        mean, rstd = Mat(1, rows, "f32"), Mat(1, rows, "f32")
        Q, E = Mat(rows, cols, "s8", pad, off), Mat(rows, -(-cols // 32), "u8", pad, off)
        done(L.gemm_layernorm_forward(rows, cols, X.ptr, X.ld, TYPES[xt], vec(gamma, pt), vec(beta, pt), TYPES[pt], EPS,
                                      Y.ptr, Y.ld, TYPES[yt], mean.ptr, rstd.ptr, Q.ptr, Q.ld, E.ptr, E.ld))
        y, m, s = R.ln_forward(x, gamma, beta, EPS)
        by, bm, bs = R.ln_forward_bounds(x, gamma, beta, EPS, yt)
        within(mean.host()[0], m, bm)
        within(rstd.host()[0], s, bs)
        within(Y.host(), y, by)
        # the checkpoint is that of y as stored, bit for bit
        q, e = R.q8_save(Y.host())
        assert np.array_equal(Q.host(), q) and np.array_equal(E.host(), e)
        assert all(a.guarded() for a in (X, Y, mean, rstd, Q, E))
        # without statistics, parameters and checkpoint: the same values for ones and zeros
        Y2 = Mat(rows, cols, yt, pad, off)
        done(L.gemm_layernorm_forward(rows, cols, X.ptr, X.ld, TYPES[xt], None, None, TYPES[pt], EPS, Y2.ptr, Y2.ld,
                                      TYPES[yt], None, None))
        one, zero = np.ones(cols), np.zeros(cols)
        within(Y2.host(), R.ln_forward(x, one, zero, EPS)[0], R.ln_forward_bounds(x, one, zero, EPS, yt)[0])
        assert Y2.guarded()


@pytest.mark.parametrize("cols", [40, 777, 4096])
def test_layernorm_forward_keeps_bad_rows_to_themselves(cols):
    """A NaN or an infinity makes its own row NaN and no other; the row's
    checkpoint blocks say so."""
    rng = np.random.default_rng(3)
    x = activations(rng, 6, cols, "bf16")
    x[1, 5], x[4, cols - 1] = np.nan, np.inf
    X, Y = Mat(6, cols, "bf16", fill=x), Mat(6, cols, "bf16")
    Q, E = Mat(6, cols, "s8"), Mat(6, -(-cols // 32), "u8")
    done(L.gemm_layernorm_forward(6, cols, X.ptr, X.ld, TYPES["bf16"], None, None, 0, EPS, Y.ptr, Y.ld, TYPES["bf16"],
                                  None, None, Q.ptr, Q.ld, E.ptr, E.ld))
    y = Y.host()
    assert np.isnan(y[[1, 4]]).all() and np.isfinite(y[[0, 2, 3, 5]]).all()
    assert (E.host()[[1, 4]] == 255).all() and (E.host()[[0, 2, 3, 5]] < 255).all() and not Q.host()[[1, 4]].any()


@pytest.mark.parametrize("rows,cols", SHAPES + [(700, 40), (2500, 128)])
@pytest.mark.parametrize("xt,gt,ot,pt", [("bf16", "bf16", "bf16", "bf16"), ("f32", "bf16", "f32", "f32"),
                                         ("bf16", "f32", "bf16", "f32"), ("f32", "f32", "f32", "f32"),
                                         ("q8", "bf16", "f32", "f32"), ("q8", "bf16", "bf16", "bf16"),
                                         ("q8", "f32", "bf16", "f32"), ("q8", "f32", "f32", "f32")])
def test_layernorm_backward(rows, cols, xt, gt, ot, pt):
    rng = np.random.default_rng(rows * 1000 + cols + 1)
    for pad, off in ((0, 0), (8, 0), (3, 1)):
        x = activations(rng, rows, cols, "f32" if xt == "q8" else xt)
        X = Q = E = None
        if xt == "q8":
            q, e = R.q8_save(x)
            x = R.q8_values(q, e)
            Q, E = Mat(rows, cols, "s8", pad, off, q), Mat(rows, -(-cols // 32), "u8", pad, off, e)
        else:
            X = Mat(rows, cols, xt, pad, off, x)
        gamma = as_kind(1 + 0.2 * rng.normal(size=cols), pt)
        _, m, s = R.ln_forward(x, gamma, 0, EPS)
        m, s = m.astype(np.float32), s.astype(np.float32)
        dy = rng.normal(size=(rows, cols))
        dy[rows // 3] = 0                          # a masked token
        dy = as_kind(dy, gt)
        D, O = Mat(rows, cols, gt, pad, off, dy), Mat(rows, cols, ot, pad, off)
        dg, db = Mat(1, cols, "f32"), Mat(1, cols, "f32")
        mean, rstd = vec(m, "f32"), vec(s, "f32")

        def call(O, dg, db, gamma):
            done(L.gemm_layernorm_backward(
                rows, cols, X.ptr if X else None, X.ld if X else 0, TYPES[ot], Q.ptr if Q else None, Q.ld if Q else 0,
                E.ptr if E else None, E.ld if E else 0, gamma, TYPES[pt], mean, rstd, D.ptr, D.ld, TYPES[gt], O.ptr,
                O.ld, TYPES[ot], dg.ptr if dg else None, db.ptr if db else None))
        call(O, dg, db, vec(gamma, pt))
        want = R.ln_backward(x, m, s, gamma, dy)
        bound = R.ln_backward_bounds(x, m, s, gamma, dy, ot)
        within(O.host(), want[0], bound[0])
        within(dg.host()[0], want[1], bound[1])
        within(db.host()[0], want[2], bound[2])
        assert not O.host()[rows // 3].any(), "a row without a gradient gets one"
        assert all(a.guarded() for a in (D, O, dg, db))
        # one parameter gradient, or none, and no gamma; the same bits again
        O2, dg2, db2 = Mat(rows, cols, ot, pad, off), Mat(1, cols, "f32"), Mat(1, cols, "f32")
        call(O2, dg2, None, vec(gamma, pt))
        assert torch.equal(O2.view, O.view) and torch.equal(dg2.view, dg.view)
        call(O2, None, db2, vec(gamma, pt))
        assert torch.equal(db2.view, db.view)
        call(O2, None, None, None)
        one = np.ones(cols)
        within(O2.host(), R.ln_backward(x, m, s, one, dy)[0], R.ln_backward_bounds(x, m, s, one, dy, ot)[0])


@pytest.mark.parametrize("rows,cols", [(4900, 2304), (5000, 4096), (20000, 100), (9000, 141)])
@pytest.mark.parametrize("xt,gt,ot", [("bf16", "bf16", "bf16"), ("q8", "bf16", "f32")])
def test_layernorm_backward_of_many_rows(rows, cols, xt, gt, ot):
    """Enough rows that every block walks many of them, the rings go round
    several times and there are many partial sums."""
    rng = np.random.default_rng(rows + cols)
    x = rng.normal(size=(rows, cols)).astype(np.float32) * 2 + 0.5
    X = Q = E = None
    if xt == "q8":
        q = rng.integers(-127, 128, size=(rows, cols)).astype(np.int8)
        e = rng.integers(118, 123, size=(rows, -(-cols // 32))).astype(np.uint8)
        x = R.q8_values(q, e)
        Q, E = Mat(rows, cols, "s8", fill=q), Mat(rows, -(-cols // 32), "u8", fill=e)
    else:
        x = as_kind(x, xt)
        X = Mat(rows, cols, xt, fill=x)
    gamma = as_kind(1 + 0.2 * rng.normal(size=cols), "f32")
    _, m, s = R.ln_forward(x, gamma, 0, EPS)
    m, s = m.astype(np.float32), s.astype(np.float32)
    dy = as_kind(rng.normal(size=(rows, cols)), gt)
    D, O = Mat(rows, cols, gt, fill=dy), Mat(rows, cols, ot)
    dg, db = Mat(1, cols, "f32"), Mat(1, cols, "f32")
    for _ in range(2):
        done(L.gemm_layernorm_backward(
            rows, cols, X.ptr if X else None, cols if X else 0, TYPES[ot], Q.ptr if Q else None, cols,
            E.ptr if E else None, E.ld if E else 0, vec(gamma, "f32"), TYPES["f32"], vec(m, "f32"), vec(s, "f32"), D.ptr,
            cols, TYPES[gt], O.ptr, cols, TYPES[ot], dg.ptr, db.ptr))
        want = R.ln_backward(x, m, s, gamma, dy)
        bound = R.ln_backward_bounds(x, m, s, gamma, dy, ot)
        within(O.host(), want[0], bound[0])
        within(dg.host()[0], want[1], bound[1])
        within(db.host()[0], want[2], bound[2])
    assert all(a.guarded() for a in (D, O, dg, db))


@pytest.mark.parametrize("rows,cols,xt", [(5000, 1024, "bf16"), (3000, 130, "bf16"), (4000, 500, "f32")])
def test_layernorm_forward_of_many_rows(rows, cols, xt):
    rng = np.random.default_rng(rows + cols)
    x = as_kind(rng.normal(size=(rows, cols)) * 3 - 1, xt)
    gamma, beta = as_kind(1 + 0.2 * rng.normal(size=cols), "bf16"), as_kind(0.2 * rng.normal(size=cols), "bf16")
    X, Y = Mat(rows, cols, xt, fill=x), Mat(rows, cols, "bf16")
    Q, E = Mat(rows, cols, "s8"), Mat(rows, -(-cols // 32), "u8")
    mean, rstd = Mat(1, rows, "f32"), Mat(1, rows, "f32")
    done(L.gemm_layernorm_forward(rows, cols, X.ptr, cols, TYPES[xt], vec(gamma, "bf16"), vec(beta, "bf16"),
                                  TYPES["bf16"], EPS, Y.ptr, cols, TYPES["bf16"], mean.ptr, rstd.ptr, Q.ptr, cols,
                                  E.ptr, E.ld))
    y, m, s = R.ln_forward(x, gamma, beta, EPS)
    by, bm, bs = R.ln_forward_bounds(x, gamma, beta, EPS, "bf16")
    within(Y.host(), y, by)
    within(mean.host()[0], m, bm)
    within(rstd.host()[0], s, bs)
    # the checkpoint's values, against those of y as stored (the blocks are
    # independent, so a sample of rows goes through the definition)
    pick = np.r_[0:50, rows - 50:rows]
    q, e = R.q8_save(Y.host()[pick])
    assert np.array_equal(Q.host()[pick], q) and np.array_equal(E.host()[pick], e)
    B = Mat(rows, cols, "f32")
    done(L.gemm_q8_restore(rows, cols, Q.ptr, cols, E.ptr, E.ld, B.ptr, cols, TYPES["f32"]))
    top = np.repeat(np.maximum.reduceat(np.abs(Y.host()), np.arange(0, cols, 32), axis=1), 32, axis=1)[:, :cols]
    assert (np.abs(B.host() - Y.host()) <= top / 126).all()
    assert all(a.guarded() for a in (X, Y, Q, E, mean, rstd))


def test_layernorm_backward_of_no_rows_is_zero():
    dg, db = torch.full((50,), 7.0, device="cuda"), torch.full((50,), 7.0, device="cuda")
    done(L.gemm_layernorm_backward(0, 50, None, 0, 0, None, 0, None, 0, None, 0, None, None, None, 0, 0, None, 0, 0,
                                   dg, db))
    assert not dg.any() and not db.any()


def hard_blocks(rng, rows, cols, kind):
    """Values of every size: exponents over the whole range, boundaries of the
    block exponent, ties, subnormals, zeros, and blocks with NaN or infinity."""
    x = rng.normal(size=(rows, cols)).astype(np.float32)
    x *= np.exp2(rng.integers(-30, 30, size=(rows, 1))).astype(np.float32)
    flat = x.reshape(-1)
    special = np.array([127, 127.5, 128, 63.5, -127, 0.5, 1.5, -2.5, 0, -0.0, 3.4e38, -3.3e38, 1e-38, 1e-40, -3e-45,
                        2.0 ** -126, 127 * 2.0 ** -126, 254 * 2.0 ** -126], np.float32)
    at = rng.integers(0, flat.size, size=max(1, flat.size // 40))
    flat[at] = special[rng.integers(0, special.size, at.size)]
    if rows > 3:
        x[1] = 0
        x[2] = special[np.arange(cols) % special.size]
        x[3, cols // 2] = np.nan
        x[3, 0] = -np.inf
    return as_kind(x, kind)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_checkpoint(rows, cols, kind):
    rng = np.random.default_rng(rows + cols)
    for pad, off in ((0, 0), (16, 0), (8, 8), (3, 1)):
        x = hard_blocks(rng, rows, cols, kind)
        X = Mat(rows, cols, kind, pad, off, x)
        Q, E = Mat(rows, cols, "s8", pad, off), Mat(rows, -(-cols // 32), "u8", pad, off)
        done(L.gemm_q8_save(rows, cols, X.ptr, X.ld, TYPES[kind], Q.ptr, Q.ld, E.ptr, E.ld))
        q, e = R.q8_save(x)
        assert np.array_equal(E.host(), e) and np.array_equal(Q.host(), q)
        values = R.q8_values(q, e)
        for back in ("bf16", "f32"):
            B = Mat(rows, cols, back, pad, off)
            done(L.gemm_q8_restore(rows, cols, Q.ptr, Q.ld, E.ptr, E.ld, B.ptr, B.ld, TYPES[back]))
            assert np.array_equal(B.host().astype(np.float64), values, equal_nan=True)
            assert B.guarded()
        assert all(a.guarded() for a in (X, Q, E))


def test_checkpoint_of_every_byte_and_exponent():
    """restore on all 256 bytes under each exponent whose values are finite."""
    e = np.arange(1, 248, dtype=np.uint8)[:, None].repeat(8, 1)       # -128 * 2^121 is past float32
    q = np.arange(-128, 128, dtype=np.int16).astype(np.int8)[None].repeat(247, 0)
    Q, E = Mat(247, 256, "s8", fill=q), Mat(247, 8, "u8", fill=e)
    for back in ("bf16", "f32"):
        B = Mat(247, 256, back)
        done(L.gemm_q8_restore(247, 256, Q.ptr, 256, E.ptr, 8, B.ptr, 256, TYPES[back]))
        assert np.array_equal(B.host().astype(np.float64), R.q8_values(q, e))


WGRAD = [(1, 1, 1), (1, 64, 64), (2, 5, 300), (63, 128, 128), (64, 129, 65), (65, 300, 1), (128, 1, 500),
         (100, 777, 333), (1000, 256, 512), (777, 500, 1501), (4096, 64, 64), (1025, 640, 384), (300, 2048, 1024),
         (6000, 130, 260), (2048, 2500, 2304)]


@pytest.mark.parametrize("T,K,N", WGRAD)
@pytest.mark.parametrize("wt", ["f32", "bf16"])
@pytest.mark.parametrize("nk", [False, True])
def test_weight_grad(T, K, N, wt, nk):
    rng = np.random.default_rng(T + 7 * K + 13 * N)
    layout = L.GEMM_B_COL_MAJOR_NxK if nk else L.GEMM_B_ROW_MAJOR_KxN
    shape = (N, K) if nk else (K, N)
    for pad, off, with_base in ((0, 0, False), (8, 0, True), (3, 1, True), (16, 8, False)):
        q, e = R.q8_save(as_kind(activations(rng, T, K, "bf16"), "bf16")) if T * K < 200000 else (
            rng.integers(-127, 128, size=(T, K)).astype(np.int8),
            rng.integers(110, 130, size=(T, -(-K // 32))).astype(np.uint8))
        dy = rng.normal(size=(T, N))
        dy[T // 2] = 0
        dy = as_kind(dy, "bf16")
        Q, E = Mat(T, K, "s8", pad, off, q), Mat(T, -(-K // 32), "u8", pad, off, e)
        D, W = Mat(T, N, "bf16", pad, off, dy), Mat(*shape, wt, pad, off)
        base = as_kind(10 * rng.normal(size=shape), wt) if with_base else None
        B = Mat(*shape, wt, pad, off, base) if with_base else None
        done(L.gemm_q8_weight_grad(T, K, N, Q.ptr, Q.ld, E.ptr, E.ld, D.ptr, D.ld, B.ptr if B else None,
                                   B.ld if B else 0, W.ptr, W.ld, layout, TYPES[wt]))
        ref, mag = R.weight_grad(R.q8_values(q, e), dy, base, nk)
        within(W.host(), ref, R.weight_grad_bound(ref, mag, wt))
        assert all(a.guarded() for a in (Q, E, D, W))
        if with_base:  # in place: the same bits
            done(L.gemm_q8_weight_grad(T, K, N, Q.ptr, Q.ld, E.ptr, E.ld, D.ptr, D.ld, B.ptr, B.ld, B.ptr, B.ld,
                                       layout, TYPES[wt]))
            assert torch.equal(B.view, W.view) and B.guarded()


@pytest.mark.parametrize("nk", [False, True])
def test_weight_grad_of_integers_is_exact(nk):
    """Small integers: every sum is below 2^24, so the float32 result is the
    integer itself, whatever the order of the additions."""
    rng = np.random.default_rng(5)
    T, K, N = 3000, 320, 448
    q = rng.integers(-8, 9, size=(T, K)).astype(np.int8)
    e = rng.integers(126, 129, size=(T, K // 32)).astype(np.uint8)      # scales 1/2, 1 and 2
    dy = rng.integers(-4, 5, size=(T, N)).astype(np.float32)
    Q, E, D = Mat(T, K, "s8", fill=q), Mat(T, K // 32, "u8", fill=e), Mat(T, N, "bf16", fill=dy)
    W = Mat(*((N, K) if nk else (K, N)), "f32")
    done(L.gemm_q8_weight_grad(T, K, N, Q.ptr, K, E.ptr, K // 32, D.ptr, N, None, 0, W.ptr, W.ld,
                               L.GEMM_B_COL_MAJOR_NxK if nk else L.GEMM_B_ROW_MAJOR_KxN, L.GEMM_TYPE_F32))
    want = R.q8_values(q, e).T @ dy.astype(np.float64)
    assert np.array_equal(W.host().astype(np.float64), want.T if nk else want)


def test_weight_grad_nan_stays_in_its_block():
    """A NaN block of the checkpoint reaches the 32 rows of dW it feeds, no others."""
    rng = np.random.default_rng(6)
    T, K, N = 200, 128, 192
    q = rng.integers(-127, 128, size=(T, K)).astype(np.int8)
    e = np.full((T, 4), 120, np.uint8)
    e[17, 2], q[17, 64:96] = 255, 0
    dy = as_kind(rng.normal(size=(T, N)), "bf16")
    Q, E, D, W = Mat(T, K, "s8", fill=q), Mat(T, 4, "u8", fill=e), Mat(T, N, "bf16", fill=dy), Mat(K, N, "f32")
    done(L.gemm_q8_weight_grad(T, K, N, Q.ptr, K, E.ptr, 4, D.ptr, N, None, 0, W.ptr, N, L.GEMM_B_ROW_MAJOR_KxN,
                               L.GEMM_TYPE_F32))
    w = W.host()
    assert np.isnan(w[64:96]).all() and np.isfinite(w[:64]).all() and np.isfinite(w[96:]).all()


@pytest.mark.parametrize("wt", ["f32", "bf16"])
def test_weight_grad_of_no_tokens_is_the_base(wt):
    base = as_kind(np.random.default_rng(2).normal(size=(70, 45)), wt)
    for pad, off in ((0, 0), (3, 1)):
        B, W = Mat(70, 45, wt, pad, off, base), Mat(70, 45, wt, pad, off)
        for src in (B, None):
            done(L.gemm_q8_weight_grad(0, 70, 45, None, 0, None, 0, None, 0, src.ptr if src else None,
                                       src.ld if src else 0, W.ptr, W.ld, L.GEMM_B_ROW_MAJOR_KxN, TYPES[wt]))
            assert np.array_equal(W.host(), base if src else np.zeros_like(base)) and W.guarded()
        done(L.gemm_q8_weight_grad(0, 70, 45, None, 0, None, 0, None, 0, B.ptr, B.ld, B.ptr, B.ld,
                                   L.GEMM_B_ROW_MAJOR_KxN, TYPES[wt]))
        assert np.array_equal(B.host(), base)


def test_same_bits_from_run_to_run_and_on_concurrent_streams():
    """Two streams run the backward pass and the weight gradient at once, many
    times; every result has the bits of the first."""
    rng = np.random.default_rng(8)
    rows, cols, n = 1500, 1024, 640
    x = activations(rng, rows, cols, "bf16")
    q, e = R.q8_save(x[:200])
    q, e = np.tile(q, (8, 1))[:rows], np.tile(e, (8, 1))[:rows]
    _, m, s = R.ln_forward(x, 1.0, 0.0, EPS)
    X, Q, E = Mat(rows, cols, "bf16", fill=x), Mat(rows, cols, "s8", fill=q), Mat(rows, cols // 32, "u8", fill=e)
    D = Mat(rows, cols, "bf16", fill=as_kind(rng.normal(size=(rows, cols)), "bf16"))
    GR = Mat(rows, n, "bf16", fill=as_kind(rng.normal(size=(rows, n)), "bf16"))
    mean, rstd = vec(m, "f32"), vec(s, "f32")
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for k in range(12):
        st = streams[k % 2]
        o = (Mat(rows, cols, "bf16"), Mat(1, cols, "f32"), Mat(1, cols, "f32"), Mat(cols, n, "f32"))
        torch.cuda.synchronize() if k < 2 else None
        outs.append(o)
    torch.cuda.synchronize()
    for k, o in enumerate(outs):
        st = streams[k % 2]
        assert L.gemm_layernorm_backward(rows, cols, X.ptr, cols, 1, None, 0, None, 0, None, 0, mean, rstd, D.ptr,
                                         cols, 1, o[0].ptr, cols, 1, o[1].ptr, o[2].ptr, stream=st) == G.GEMM_OK
        assert L.gemm_q8_weight_grad(rows, cols, n, Q.ptr, cols, E.ptr, cols // 32, GR.ptr, n, None, 0, o[3].ptr, n,
                                     L.GEMM_B_ROW_MAJOR_KxN, 0, stream=st) == G.GEMM_OK
    torch.cuda.synchronize()
    assert G.gemm_device_status() == G.GEMM_OK
    for o in outs[1:]:
        for a, b in zip(o, outs[0]):
            assert torch.equal(a.view, b.view)


def test_graph_capture_replays_with_new_inputs():
    """A training step's calls captured once and replayed on other inputs."""
    rng = np.random.default_rng(9)
    rows, cols, n = 500, 768, 512
    X, Y = Mat(rows, cols, "bf16"), Mat(rows, cols, "bf16")
    Q, E = Mat(rows, cols, "s8"), Mat(rows, cols // 32, "u8")
    D, GR = Mat(rows, cols, "bf16"), Mat(rows, n, "bf16")
    mean, rstd = Mat(1, rows, "f32"), Mat(1, rows, "f32")
    DX, dg, db, W = Mat(rows, cols, "bf16"), Mat(1, cols, "f32"), Mat(1, cols, "f32"), Mat(cols, n, "f32")
    st = torch.cuda.Stream()

    def step():
        for s in (
            L.gemm_layernorm_forward(rows, cols, X.ptr, cols, 1, None, None, 0, EPS, Y.ptr, cols, 1, mean.ptr, rstd.ptr,
                                     Q.ptr, cols, E.ptr, cols // 32, stream=st),
            L.gemm_q8_weight_grad(rows, cols, n, Q.ptr, cols, E.ptr, cols // 32, GR.ptr, n, None, 0, W.ptr, n,
                                  L.GEMM_B_ROW_MAJOR_KxN, 0, stream=st),
            L.gemm_layernorm_backward(rows, cols, X.ptr, cols, 1, None, 0, None, 0, None, 0, mean.ptr, rstd.ptr, D.ptr,
                                      cols, 1, DX.ptr, cols, 1, dg.ptr, db.ptr, stream=st)):
            assert s == G.GEMM_OK, G.gemm_status_string(s)

    def refill():
        for M in (X, D, GR):
            M.view.copy_(torch.from_numpy(rng.normal(size=M.view.shape)).float())
        torch.cuda.synchronize()

    refill()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        step()
    outs = (Y, Q, E, mean, rstd, DX, dg, db, W)
    for _ in range(3):
        refill()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        got = [o.view.clone() for o in outs]
        step()
        torch.cuda.synchronize()
        for a, o in zip(got, outs):
            assert torch.equal(a, o.view)


def test_offsets_past_32_bits():
    """A checkpoint and an activation whose last rows lie past 2^31 elements
    (a pitch far above the width)."""
    rng = np.random.default_rng(10)
    cols, ld, rows = 100, (1 << 20) + 8, 2100             # 2100 * 2^20 > 2^31 elements
    buf = torch.zeros(rows * ld, dtype=torch.int8, device="cuda")
    x = as_kind(rng.normal(size=(rows, cols)), "bf16")
    X, E, B = Mat(rows, cols, "bf16", fill=x), Mat(rows, 4, "u8"), Mat(rows, cols, "f32")
    done(L.gemm_q8_save(rows, cols, X.ptr, cols, 1, buf, ld, E.ptr, 4))
    done(L.gemm_q8_restore(rows, cols, buf, ld, E.ptr, 4, B.ptr, cols, 0))
    assert np.array_equal(B.host().astype(np.float64), R.q8_values(*R.q8_save(x)))
