"""Coverage of the reduction and the workspace of exfold_linear_forward's plans, with the length that copied rows are
padded to computed here: the splits end exactly behind it, and the workspace holds every region at its 256-byte
alignment, for rows of x on or off 16 bytes."""

import ctypes
import random

from paper_2608_24938_amd import exfold as X

from .linear_builds import RING, TILE, WIDE, plan

ALIGN = 256


def region(size):
    return -(-size // ALIGN) * ALIGN


def padded(k, esz):
    """The length of a copied row: as it is where it holds whole 16-byte pieces, else whole stages of 128 bytes."""
    return k if k * esz % 16 == 0 else -(-k * esz // 128) * 128 // esz


def size_of(m, n, k, bf16, gated, ldw):
    dtype = X.BF16 if bf16 else X.F32
    ls = X._Linear(k, n, ldw, 1 << 20, None, dtype, dtype, 0, int(gated))
    return X.lib().exfold_linear_workspace_size(ctypes.byref(ls), m)


def draws(seed, count):
    rng = random.Random(seed)
    for _ in range(count):
        bf16, gated = rng.random() < 0.6, rng.random() < 0.5
        m, n, k = (int(2 ** rng.uniform(0, e)) for e in (13, 14, 14))
        if rng.random() < 0.5:
            k = max(8, k // 8 * 8)
        yield m, n, k, bf16, gated, k + rng.choice((0, 0, 8, 3, 1))


def test_splits_end_behind_the_reduction():
    seen = set()
    for m, n, k, bf16, gated, ldw in draws(11, 4000):
        esz = 2 if bf16 else 4
        for aligned in (True, False):
            p = plan(m, n, k, bf16, gated, aligned, ldw)
            run = padded(k, esz) if p["copy_x"] or p["copy_w"] else k
            assert p["kc"] * (p["ksplit"] - 1) < run <= p["kc"] * p["ksplit"], (m, n, k, bf16, gated, ldw, aligned, p)
            if p["ksplit"] > 1:
                assert p["kc"] * esz % 128 == 0
            if p["kind"] == WIDE:
                assert run * esz % 128 == 0 and run * esz >= 256 and p["ksplit"] == 1
            if p["kind"] == RING:
                assert run * esz % 16 == 0
            if p["kind"] == TILE:
                assert not (p["copy_x"] or p["copy_w"])
            seen.add((p["kind"], p["ksplit"] > 1, p["copy_x"], p["copy_w"]))
    assert {(RING, True, 1, 1), (RING, False, 1, 0), (RING, False, 0, 1), (TILE, True, 0, 0), (WIDE, False, 1, 1)} <= seen


def test_workspace_holds_the_copies_and_the_partial_sums():
    for m, n, k, bf16, gated, ldw in draws(12, 4000):
        esz, rows = 2 if bf16 else 4, 2 * n if gated else n
        need = []
        for aligned in (True, False):
            p = plan(m, n, k, bf16, gated, aligned, ldw)
            kp = padded(k, esz)
            parts = p["ksplit"] * m * -(-n // 4) * 4 * (rows // n) * 4 if p["ksplit"] > 1 else 0
            need.append(region(m * kp * esz if p["copy_x"] else 0) + region(rows * kp * esz if p["copy_w"] else 0) + region(parts))
        assert size_of(m, n, k, bf16, gated, ldw) == max(need), (m, n, k, bf16, gated, ldw, need)


def test_fewer_rows_may_need_more():
    # as the header says: the size is that of exactly these rows
    sizes = {m: size_of(m, 4096, 14336, True, False, 14336) for m in (1, 32, 64, 100, 128, 4096)}
    assert sizes[1] == 0 and sizes[64] > sizes[100] > 0
    # rows of x off 16 bytes are what 4096 rows need it for
    assert sizes[4096] == region(4096 * 14336 * 2) and plan(4096, 4096, 14336)["copy_x"] == 0
