"""Which build of a kernel a call of exfold_linear_forward launches, from the host query of its plan: the tests
that are there for one build assert that they reach it."""

import ctypes

from paper_2608_24938_amd import exfold as X

FEW, TILE, RING, WIDE = range(4)


def plan(m, n, k, bf16=True, gated=False, x_aligned=True, ldw=None, cu=256):
    dtype = X.BF16 if bf16 else X.F32
    ls = X._Linear(k, n, ldw or k, 1 << 20, None, dtype, dtype, 0, int(gated))
    out = (ctypes.c_int32 * 8)()
    assert X.lib().exfold_linear_plan(ctypes.byref(ls), m, int(x_aligned), cu, out) == X.OK
    return dict(zip(("kind", "bm", "bn", "ksplit", "kc", "grid", "copy_x", "copy_w"), out))


def build(m, n, k, bf16=True, gated=False, x_aligned=True, ldw=None, cu=256):
    """(family, what tells its builds apart ...) of the call's product kernel, with "split" where partial sums are joined."""
    p = plan(m, n, k, bf16, gated, x_aligned, ldw, cu)
    esz = 2 if bf16 else 4
    split = ("split",) if p["ksplit"] > 1 else ()
    if p["kind"] == FEW:
        vec = x_aligned and (ldw or k) * esz % 16 == 0 and k * esz % 16 == 0
        return ("few", p["bm"], p["bn"], "pieces" if vec else "any")
    if p["kind"] == WIDE:
        return ("wide",)
    if p["kind"] == TILE:
        return ("tile",) + split
    if p["bm"] == 128:
        kind = 2 if p["grid"] > cu or not bf16 else 4              # buffers of the ring
    elif p["bn"] == 128:
        kind = 2 if p["kc"] * esz <= 256 else 3
    else:
        kind = "once" if m <= p["bm"] else "again"                 # how the weights are loaded
    return ("ring", p["bm"], p["bn"], kind) + split
