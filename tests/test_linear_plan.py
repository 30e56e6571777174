"""Plans of exfold_linear_forward (host logic, no GPU): the kernel family of each kind of call, grids that
cover every output and splits that cover the reduction exactly once, and the workspace they need."""

import ctypes
import random

import pytest

from paper_2608_24938_amd import exfold as X

FEW, TILE, RING, WIDE = range(4)
W = 1 << 20     # weights are never dereferenced by the planner


def plan(m, n, k, dtype=X.BF16, gated=False, x_aligned=True, ldw=None, cu=256):
    ls = X._Linear(k, n, ldw or k, W, None, dtype, dtype, 0, int(gated))
    out = (ctypes.c_int32 * 8)()
    assert X.lib().exfold_linear_plan(ctypes.byref(ls), m, int(x_aligned), cu, out) == X.OK
    return dict(zip(("kind", "bm", "bn", "ksplit", "kc", "grid", "copy_x", "copy_w"), out)), ls


@pytest.mark.parametrize("args,kw,kind", [
    ((1, 128, 2048), {}, FEW), ((4, 28672, 4096), {}, FEW), ((1, 7, 13), {}, FEW),
    ((5000, 1, 2056), {}, FEW), ((16, 128, 2048), {}, FEW), ((66000, 2, 2048), {}, RING),
    ((32, 4096, 14336), {}, RING), ((64, 28672, 4096), {}, RING), ((600, 2048, 768), dict(dtype=X.F32), RING),
    ((1237, 1408, 4096), dict(gated=True), RING), ((8192, 14336, 4096), dict(gated=True), WIDE),
    ((8192, 8192, 8192), {}, WIDE), ((8192, 8192, 8192), dict(dtype=X.F32), RING),
    ((8192, 8192, 8200), {}, RING),                            # not whole stages: no wide tile
    ((30, 14001, 4001), {}, TILE), ((2000, 8001, 8001), {}, WIDE),   # copied to whole stages
])
def test_kernel_family(args, kw, kind):
    p, _ = plan(*args, **kw)
    assert p["kind"] == kind, p


def test_rows_off_alignment_are_copied_where_they_are_large():
    p, _ = plan(2000, 8001, 8001, ldw=8004)
    assert (p["copy_x"], p["copy_w"]) == (1, 1)                # no whole pieces: both, with zeros behind
    p, _ = plan(4000, 4096, 4096, x_aligned=False)
    assert (p["copy_x"], p["copy_w"]) == (1, 0)                # only x starts elsewhere
    p, _ = plan(4000, 4096, 4096, ldw=4099)
    assert (p["copy_x"], p["copy_w"]) == (0, 1)
    assert plan(4000, 4096, 4096)[0]["copy_x"] == 0


def test_every_plan_covers_its_outputs_and_its_reduction():
    rng = random.Random(1)
    for _ in range(3000):
        dtype, gated, cu = rng.choice((X.BF16, X.F32)), rng.random() < 0.5, rng.choice((256, 256, 64, 1, 304))
        m, n, k = (int(2 ** rng.uniform(0, e)) for e in (13, 14, 14))
        if rng.random() < 0.5:
            k = max(8, k // 8 * 8)
        aligned = rng.random() < 0.7
        p, ls = plan(m, n, k, dtype, gated, aligned, k + rng.choice((0, 0, 8, 3)), cu)
        cols = p["bn"] // 2 if gated else p["bn"]
        tiles = -(-m // p["bm"]) * -(-n // cols)
        assert p["grid"] == tiles * p["ksplit"] and p["grid"] > 0
        run = k if not (p["copy_x"] and p["copy_w"]) else p["kc"] * p["ksplit"]
        assert p["kc"] * (p["ksplit"] - 1) < run <= p["kc"] * p["ksplit"], p    # the last split is not empty
        esz = 2 if dtype == X.BF16 else 4
        pieces = k * esz % 16 == 0
        if p["kind"] in (RING, WIDE):
            assert aligned or p["copy_x"]
            assert (pieces and ls.ldw * esz % 16 == 0) or p["copy_w"]
            assert pieces or (p["copy_x"] and p["copy_w"])
        if p["ksplit"] > 1:
            assert p["kc"] * esz % 128 == 0                                   # whole stages
        if cu == 256:
            size = X.lib().exfold_linear_workspace_size(ctypes.byref(ls), m)
            part = p["ksplit"] * m * -(-n // 4) * 4 * (2 if gated else 1) * 4 if p["ksplit"] > 1 else 0
            rows = (m if p["copy_x"] else 0) + (n * (2 if gated else 1) if p["copy_w"] else 0)
            assert size >= part + rows * k * esz


def test_query_refusals():
    _, ls = plan(8, 8, 8)
    out = (ctypes.c_int32 * 8)()
    q = X.lib().exfold_linear_plan
    assert q(ctypes.byref(ls), 0, 1, 256, out) == X.ERR_SHAPE
    assert q(ctypes.byref(ls), 8, 1, 0, out) == X.ERR_SHAPE
    assert q(ctypes.byref(ls), 8, 1, 256, None) == X.ERR_NULL
    assert q(None, 8, 1, 256, out) == X.ERR_NULL
    ls.act = 9
    assert q(ctypes.byref(ls), 8, 1, 256, out) == X.ERR_ARG
