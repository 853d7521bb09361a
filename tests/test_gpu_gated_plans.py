"""Every compiled tile of the gated feed-forward block's tensor-core kernel in
every way that its plans use it -- one round, several, a split tail alone and
after whole rounds -- by the planner's overrides, whose effect is read from the
plan that the library prints.  In both layouts, on aligned rows, rows whose
checkpoint starts on 8 bytes and rows that start anywhere, against the 64-bit
definition."""
import functools
import re

import numpy as np
import pytest
import torch

from paper_2512_13282_gb300 import gemm as G
from paper_2512_13282_gb300 import layer as L
from tests import gated_ref as A
from tests.test_gpu_gated import ACT, KN, NAMES, NK, bf, gate_inputs, run_backward, run_forward, weight
from tests.test_gpu_layer import Mat, _lib, within  # noqa: F401

pytestmark = pytest.mark.gpu

# tile: (CTA pair, accumulator columns); rows and features of its tiles
FORWARD = {(1, 256): (256, 128), (0, 128): (128, 64)}
BACKWARD = {(1, 256): (256, 256), (0, 128): (128, 128), (0, 64): (128, 64)}
K = 520                       # nine k-blocks, the last of eight columns
# alignment: features short of the largest problem's, pitch and base offset; in place
PLACES = {"on 16": (8, 0, 0, True), "checkpoint on 8": (0, 8, 8, False), "anywhere": (19, 3, 1, True)}


def size(tile_m, tile_f, pair, full):
    """A problem of a round and a few tiles, with a broken last row and column of them, or of
    four tiles."""
    if not full:
        return 2 * tile_m - 31, tile_f + 72
    slots = torch.cuda.get_device_properties(0).multi_processor_count // (2 if pair else 1)
    tn = int(slots ** 0.5) + 1
    tm = slots // tn + 1
    assert slots < tm * tn < 1.5 * slots
    return tm * tile_m - 31, (tn - 1) * tile_f + 24


def force(monkeypatch, tile, splits):
    for name, value in (("PAIR", tile[0]), ("BN", tile[1]), ("TAIL_SPLITS", splits), ("DEBUG", 1)):
        monkeypatch.setenv(f"GB300_GEMM_{name}", str(value))
    G.gemm_reload_overrides()


def planned(capfd, tile, splits, full):
    """The plan printed last is the one forced."""
    line = [s for s in capfd.readouterr().err.splitlines() if "gated" in s][-1]
    kind, bn, tm, tn, whole, split = re.search(r": (\w+) (\d+), (\d+)x(\d+) tiles, (\d+) in whole, tail split in (\d+)",
                                               line).groups()
    assert (kind == "pair", int(bn), int(split)) == (bool(tile[0]), tile[1], splits), line
    assert int(tm) * int(tn) > int(whole) if splits else int(tm) * int(tn) == int(whole), line
    assert (int(whole) > 4) == full if splits else True, line


@functools.lru_cache(maxsize=4)
def forward_problem(T, F):
    rng = np.random.default_rng(T + F)
    x, wg, wu = bf(rng.normal(size=(T, K))), *(bf(rng.normal(size=(K, F)) / K ** 0.5) for _ in range(2))
    return x, wg, wu, A.forward(x, wg, wu, "silu")


@functools.lru_cache(maxsize=4)
def backward_problem(T, F):
    rng = np.random.default_rng(T + F)
    g, u = gate_inputs(rng, T, F)
    d, wd = bf(1e-2 * rng.normal(size=(T, K))), bf(rng.normal(size=(F, K)) / K ** 0.5)
    return g, u, d, wd, A.backward(*A.product(d, wd.T), g, u, "gelu")


def cases(tiles):
    return [pytest.param(tile, splits, full, id=f"{'pair' if tile[0] else 'single'} {tile[1]} "
                         f"{'rounds' if full else 'one round'}{f' split in {splits}' if splits else ''}")
            for tile in tiles for full in (False, True) for splits in (0, 2)]


@pytest.mark.parametrize("tile,splits,full", cases(FORWARD))
def test_forward(tile, splits, full, monkeypatch, capfd):
    T, most = size(*FORWARD[tile], tile[0], full)
    force(monkeypatch, tile, splits)
    for fewer, pad, off, keep in PLACES.values():
        F = most - fewer
        x, wg, wu, want = forward_problem(T, most)
        for layout in (KN, NK):
            capfd.readouterr()
            got = run_forward(x, wg[:, :F], wu[:, :F], "silu", layout, pad, off, keep)
            planned(capfd, tile, splits, full)
            for m, (w, bound) in zip(got, want):
                within(m, w[:, :F], bound[:, :F])


@pytest.mark.parametrize("tile,splits,full", cases(BACKWARD))
def test_backward(tile, splits, full, monkeypatch, capfd):
    T, most = size(*BACKWARD[tile], tile[0], full)
    force(monkeypatch, tile, splits)
    for fewer, pad, off, in_place in PLACES.values():
        F = most - fewer
        g, u, d, wd, want = backward_problem(T, most)
        dg, du, h = [(v[:, :F], e[:, :F]) for v, e in want]
        for layout in (KN, NK):
            D, W = Mat(T, K, "bf16", pad, off, d), weight(wd[:F], layout, pad, off)
            capfd.readouterr()
            got, ck = run_backward(g[:, :F], u[:, :F], "gelu", True, lambda *a: L.gemm_gated_down_backward(
                T, K, F, D.ptr, D.ld, W.ptr, W.ld, layout, *a), pad, off, in_place)
            planned(capfd, tile, splits, full)
            within(got[0], *dg)
            within(got[1], *du)
            assert A.held_ok(*ck, *h) and D.guarded() and W.guarded()


@pytest.mark.parametrize("tile", BACKWARD)
def test_rounds_with_a_tail_repeat_bit_for_bit(tile, monkeypatch):
    T, F = size(*BACKWARD[tile], tile[0], True)
    force(monkeypatch, tile, 2)
    monkeypatch.delenv("GB300_GEMM_DEBUG")
    g, u, d, wd, _ = backward_problem(T, F)
    D, W = Mat(T, K, "bf16", fill=d), weight(wd, KN)
    runs = [run_backward(g, u, "gelu", True, lambda *a: L.gemm_gated_down_backward(
        T, K, F, D.ptr, D.ld, W.ptr, W.ld, KN, *a)) for _ in range(3)]
    for got, ck in runs[1:]:
        assert all(np.array_equal(a, b) for a, b in zip(runs[0][0] + list(runs[0][1]), got + list(ck)))


def test_what_is_not_compiled_is_not_forced(monkeypatch, capfd):
    """An accumulator width or a family without a tile, a tail with nothing to
    split: the planner's choice of the rest."""
    x, wg, wu, want = forward_problem(100, 64)
    for name, value in (("BN", 192), ("PAIR", 1), ("TAIL_SPLITS", 16)):
        with monkeypatch.context() as m:
            m.setenv(f"GB300_GEMM_{name}", str(value))
            G.gemm_reload_overrides()
            for got, (w, bound) in zip(run_forward(x, wg, wu, "silu", KN), want):
                within(got, w, bound)
