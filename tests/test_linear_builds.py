"""Every build of the matrix product's kernels runs: one call for each, at a size whose plan is asserted to launch it.
The sizes leave rows, columns and pieces over, turn the ring's buffers at least once and end splits inside a stage."""

import pytest
import torch

from paper_2608_24938_amd import exfold as X

from .gpu_common import DEV, sync
from .linear_builds import build
from .test_gpu_linear import compare

# M, N, K, bf16, gated, rows of x on 16 bytes, rows of w on 16 bytes, the build
CASES = [
    # bf16, gated
    (1, 13, 4615, 1, 1, 1, 0, "few-1-2-any"), (1, 13, 4536, 1, 1, 1, 1, "few-1-2-pieces"),
    (1, 2096, 502, 1, 1, 0, 0, "few-1-8-any"), (1, 2196, 560, 1, 1, 1, 1, "few-1-8-pieces"),
    (2, 13, 4506, 1, 1, 1, 1, "few-2-2-any"), (2, 13, 4536, 1, 1, 1, 1, "few-2-2-pieces"),
    (2, 2092, 545, 1, 1, 1, 1, "few-2-8-any"), (2, 2064, 536, 1, 1, 1, 1, "few-2-8-pieces"),
    (3, 13, 503, 1, 1, 0, 1, "few-4-2-any"), (3, 13, 512, 1, 1, 1, 1, "few-4-2-pieces"),
    (3, 2144, 572, 1, 1, 0, 1, "few-4-8-any"), (4, 2106, 504, 1, 1, 1, 1, "few-4-8-pieces"),
    (1470, 2233, 392, 1, 1, 1, 1, "ring-128-128-2"), (1035, 972, 9511, 1, 1, 1, 1, "ring-128-128-2-split"),
    (1477, 694, 392, 1, 1, 1, 1, "ring-128-128-4"), (1201, 443, 4984, 1, 1, 1, 1, "ring-128-128-4-split"),
    (68, 12, 528, 1, 1, 1, 1, "ring-32-64-again"), (36, 23, 14608, 1, 1, 1, 1, "ring-32-64-again-split"),
    (30, 141, 560, 1, 1, 1, 1, "ring-32-64-once"), (23, 29, 15552, 1, 1, 1, 1, "ring-32-64-once-split"),
    (578, 817, 72, 1, 1, 1, 1, "ring-64-128-2"), (666, 794, 392, 1, 1, 1, 1, "ring-64-128-3"),
    (351, 335, 6240, 1, 1, 1, 1, "ring-64-128-3-split"), (694, 386, 384, 1, 1, 1, 1, "ring-64-64-again"),
    (406, 139, 3472, 1, 1, 1, 1, "ring-64-64-again-split"), (61, 4884, 432, 1, 1, 1, 1, "ring-64-64-once"),
    (38, 716, 4856, 1, 1, 1, 1, "ring-64-64-once-split"), (38, 287, 6491, 1, 1, 0, 0, "tile-split"),
    (706, 697, 196, 1, 1, 1, 1, "tile"), (2071, 1550, 320, 1, 1, 1, 1, "wide"),
    # bf16
    (1, 13, 4540, 1, 0, 0, 0, "few-1-2-any"), (1, 13, 4504, 1, 0, 1, 1, "few-1-2-pieces"),
    (1, 4252, 521, 1, 0, 1, 0, "few-1-8-any"), (1, 4124, 584, 1, 0, 1, 1, "few-1-8-pieces"),
    (2, 13, 4979, 1, 0, 1, 1, "few-2-2-any"), (2, 13, 4584, 1, 0, 1, 1, "few-2-2-pieces"),
    (2, 4320, 604, 1, 0, 1, 0, "few-2-8-any"), (2, 4368, 592, 1, 0, 1, 1, "few-2-8-pieces"),
    (3, 13, 507, 1, 0, 1, 0, "few-4-2-any"), (3, 13, 520, 1, 0, 1, 1, "few-4-2-pieces"),
    (3, 4488, 515, 1, 0, 0, 0, "few-4-8-any"), (3, 4104, 504, 1, 0, 1, 1, "few-4-8-pieces"),
    (3021, 2212, 392, 1, 0, 1, 1, "ring-128-128-2"), (2641, 4, 13160, 1, 0, 1, 1, "ring-128-128-2-split"),
    (927, 2556, 384, 1, 0, 1, 1, "ring-128-128-4"), (625, 1700, 5176, 1, 0, 1, 1, "ring-128-128-4-split"),
    (73, 11, 544, 1, 0, 1, 1, "ring-32-64-again"), (52, 27, 14432, 1, 0, 1, 1, "ring-32-64-again-split"),
    (31, 268, 512, 1, 0, 1, 1, "ring-32-64-once"), (28, 46, 15792, 1, 0, 1, 1, "ring-32-64-once-split"),
    (1110, 901, 72, 1, 0, 1, 1, "ring-64-128-2"), (657, 1513, 384, 1, 0, 1, 1, "ring-64-128-3"),
    (430, 796, 5120, 1, 0, 1, 1, "ring-64-128-3-split"), (654, 772, 408, 1, 0, 1, 1, "ring-64-64-again"),
    (459, 350, 2837, 1, 0, 1, 1, "ring-64-64-again-split"), (60, 8364, 400, 1, 0, 1, 1, "ring-64-64-once"),
    (45, 2060, 3352, 1, 0, 1, 1, "ring-64-64-once-split"), (171, 672, 4186, 1, 0, 0, 1, "tile-split"),
    (250, 2252, 192, 1, 0, 0, 0, "tile"), (2548, 2470, 320, 1, 0, 1, 1, "wide"),
    # float32, gated
    (1, 13, 2290, 0, 1, 1, 1, "few-1-2-any"), (1, 13, 2328, 0, 1, 1, 1, "few-1-2-pieces"),
    (1, 2132, 256, 0, 1, 0, 0, "few-1-8-any"), (1, 2220, 260, 0, 1, 1, 1, "few-1-8-pieces"),
    (2, 13, 2287, 0, 1, 1, 0, "few-2-2-any"), (2, 13, 2264, 0, 1, 1, 1, "few-2-2-pieces"),
    (2, 2248, 286, 0, 1, 0, 0, "few-2-8-any"), (2, 2215, 256, 0, 1, 1, 1, "few-2-8-pieces"),
    (3, 13, 264, 0, 1, 1, 0, "few-4-2-any"), (3, 13, 252, 0, 1, 1, 1, "few-4-2-pieces"),
    (4, 2147, 270, 0, 1, 1, 1, "few-4-8-any"), (4, 2140, 268, 0, 1, 1, 1, "few-4-8-pieces"),
    (615, 2121, 2088, 0, 1, 1, 1, "ring-128-128-2-split"), (67, 7, 180, 0, 1, 1, 1, "ring-32-64-again"),
    (68, 10, 596, 0, 1, 1, 1, "ring-32-64-again-split"), (31, 193, 164, 0, 1, 1, 1, "ring-32-64-once"),
    (29, 254, 581, 0, 1, 0, 0, "ring-32-64-once-split"), (723, 722, 36, 0, 1, 1, 1, "ring-64-128-2"),
    (554, 900, 196, 0, 1, 1, 1, "ring-64-128-3"), (367, 356, 1732, 0, 1, 1, 1, "ring-64-128-3-split"),
    (759, 324, 204, 0, 1, 1, 1, "ring-64-64-again"), (337, 244, 1424, 0, 1, 1, 1, "ring-64-64-again-split"),
    (54, 4428, 212, 0, 1, 1, 1, "ring-64-64-once"), (41, 1436, 1112, 0, 1, 1, 1, "ring-64-64-once-split"),
    (721, 744, 356, 0, 1, 1, 0, "tile-split"), (1036, 513, 98, 0, 1, 0, 0, "tile"),
    # float32
    (1, 13, 2274, 0, 0, 0, 0, "few-1-2-any"), (1, 13, 2272, 0, 0, 1, 1, "few-1-2-pieces"),
    (1, 4368, 250, 0, 0, 1, 0, "few-1-8-any"), (1, 4104, 260, 0, 0, 1, 1, "few-1-8-pieces"),
    (2, 13, 2367, 0, 0, 0, 1, "few-2-2-any"), (2, 13, 2272, 0, 0, 1, 1, "few-2-2-pieces"),
    (2, 4136, 256, 0, 0, 1, 0, "few-2-8-any"), (2, 4960, 260, 0, 0, 1, 1, "few-2-8-pieces"),
    (3, 13, 257, 0, 0, 1, 1, "few-4-2-any"), (3, 13, 256, 0, 0, 1, 1, "few-4-2-pieces"),
    (4, 4116, 275, 0, 0, 1, 0, "few-4-8-any"), (4, 4584, 260, 0, 0, 1, 1, "few-4-8-pieces"),
    (1487, 1748, 2540, 0, 0, 1, 1, "ring-128-128-2-split"), (68, 13, 160, 0, 0, 1, 1, "ring-32-64-again"),
    (77, 12, 580, 0, 0, 1, 1, "ring-32-64-again-split"), (30, 428, 183, 0, 0, 1, 0, "ring-32-64-once"),
    (26, 453, 604, 0, 0, 1, 1, "ring-32-64-once-split"), (869, 1185, 36, 0, 0, 1, 1, "ring-64-128-2"),
    (1297, 782, 224, 0, 0, 1, 1, "ring-64-128-3"), (1036, 500, 960, 0, 0, 1, 1, "ring-64-128-3-split"),
    (418, 1196, 196, 0, 0, 1, 1, "ring-64-64-again"), (350, 460, 1401, 0, 0, 0, 1, "ring-64-64-again-split"),
    (50, 8372, 226, 0, 0, 1, 1, "ring-64-64-once"), (33, 2875, 1236, 0, 0, 1, 1, "ring-64-64-once-split"),
    (1804, 532, 354, 0, 0, 0, 1, "tile-split"), (1076, 1024, 104, 0, 0, 0, 0, "tile"),
]
# rows in several groups, and few columns of many rows, on the vector units
FEW = [(10, 130, 2056, 1, 0, 1, 1, "few-4-2-pieces"), (63, 2, 515, 1, 1, 0, 0, "few-4-2-any"),
       (37, 3, 1028, 0, 0, 1, 1, "few-4-2-pieces"), (5001, 1, 2056, 1, 0, 1, 1, "few-4-2-pieces")]


def row_stride(k, esz, aligned):
    """Elements between rows of k: whole 16-byte pieces, or one element more."""
    return -(-k * esz // 16) * 16 // esz + (0 if aligned else 1)


def test_the_cases_reach_every_build():
    rings = [(bm, bn, kind) for bm, bn, kinds in ((32, 64, ("once", "again")), (64, 64, ("once", "again")), (64, 128, (3,)),
                                                  (128, 128, (2, 4))) for kind in kinds]
    few = [("few", mt, rw, vec) for mt in (1, 2, 4) for rw in (2, 8) for vec in ("pieces", "any")]
    ring = [("ring",) + r + s for r in rings for s in ((), ("split",))] + [("ring", 64, 128, 2)]
    every = few + ring + [("tile",), ("tile", "split"), ("wide",)]
    want = {(bf16, gated, "-".join(map(str, b))) for bf16 in (0, 1) for gated in (0, 1) for b in every
            # float32: no wide tiles; 128 x 128 only in splits over more than the CUs
            if bf16 or not (b == ("wide",) or b[:3] == ("ring", 128, 128) and b[3:] != (2, "split"))}
    for m, n, k, bf16, gated, xa, wa, name in CASES + FEW:
        b = build(m, n, k, bool(bf16), bool(gated), bool(xa), row_stride(k, 2 if bf16 else 4, wa))
        assert "-".join(map(str, b)) == name, (m, n, k, bf16, gated, xa, wa)
    assert {(c[3], c[4], c[7]) for c in CASES} == want


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,bf16,gated,xa,wa,name", CASES + FEW,
                         ids=lambda v: v if isinstance(v, str) else None)
def test_build(M, N, K, bf16, gated, xa, wa, name):
    cu = torch.cuda.get_device_properties(0).multi_processor_count
    dtype, rows = torch.bfloat16 if bf16 else torch.float32, 2 * N if gated else N
    esz = 2 if bf16 else 4
    g = torch.Generator().manual_seed(M * 7 + N * 3 + K)

    def cut(rr, aligned, scale):
        """K-long rows of a buffer that holds NaN behind them, one element in where they are not aligned."""
        ld, off = row_stride(K, esz, aligned), 0 if aligned else 1
        buf = torch.full((off + rr * ld,), float("nan"), dtype=dtype)
        buf[off:].view(rr, ld)[:, :K] = (torch.randn(rr, K, generator=g) * scale).to(dtype)
        return buf.to(DEV)[off:].view(rr, ld)[:, :K]

    x, w = cut(M, xa, 1.0), cut(rows, wa, 1.5 / K ** 0.5)
    ldw = row_stride(K, esz, wa)
    assert "-".join(map(str, build(M, N, K, bool(bf16), bool(gated), bool(xa), ldw, cu))) == name
    b = torch.randn(rows, generator=g).to(DEV)
    act = ("silu", "gelu", "none", "gelu_tanh", "relu")[(M + N) % 5]
    for out_dtype in [dtype, torch.float32][:2 if bf16 else 1]:
        r = torch.randn(M, N, generator=g).to(out_dtype).to(DEV)
        y = X.linear(x, w, bias=b, act=act, gated=bool(gated), residual=r, out_dtype=out_dtype)
        sync()
        compare(y, x, w, b, r, act, bool(gated))
