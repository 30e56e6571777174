"""Calls of linear as a program makes them beside the plain ones: captured without a workspace of the caller's, two
graphs in turn, gated onto its residual in place, one operand used twice."""

import pytest
import torch

from paper_2608_24938_amd import exfold as X

from .gpu_common import DEV, sync
from .linear_builds import plan
from .test_gpu_linear import compare, data

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K,gated,xpad", [(33, 512, 8192, False, 0), (40, 256, 4096, True, 0), (600, 700, 2049, False, 3),
                                              (3, 512, 4096, True, 0)])
def test_two_graphs_captured_without_a_workspace(M, N, K, gated, xpad):
    # the workspace that the binding makes in a capture belongs to that graph: two of them in turn, eager calls between
    p = plan(M, N, K, gated=gated, x_aligned=not xpad)
    assert p["ksplit"] > 1 or p["copy_x"] or M < 5
    x, w, b, r = data(M, N, K, torch.bfloat16, gated, True, True, torch.bfloat16, pad=xpad)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        X.linear(x, w, bias=b, act="gelu", gated=gated, residual=r)
    torch.cuda.current_stream().wait_stream(side)
    sync()
    graphs = []
    for act in ("gelu", "relu"):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            h = X.linear(x, w, bias=b, act=act, gated=gated, residual=r)
            y = X.linear(x, w, bias=b, act=act, gated=gated, residual=h)      # the same workspace memory, in order
        graphs.append((g, act, h, y))
    for rep in range(4):
        x.copy_(torch.randn(M, K, generator=torch.Generator().manual_seed(rep)).bfloat16())
        want = []
        for _, act, _, _ in graphs:
            eh = X.linear(x, w, bias=b, act=act, gated=gated, residual=r)
            want.append((eh, X.linear(x, w, bias=b, act=act, gated=gated, residual=eh)))
        for g, _, _, _ in graphs if rep % 2 else reversed(graphs):
            g.replay()
        sync()
        for (_, act, h, y), (eh, ey) in zip(graphs, want):
            assert torch.equal(h.view(torch.int16), eh.view(torch.int16)), f"replay {rep} {act}"
            assert torch.equal(y.view(torch.int16), ey.view(torch.int16)), f"replay {rep} {act}"
        compare(want[0][0], x, w, b, r, "gelu", gated)


@pytest.mark.parametrize("M,N,K", [(1, 256, 512), (33, 130, 8192), (70, 200, 320), (300, 90, 45), (2071, 1550, 320)])
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_gated_onto_its_residual_in_place(M, N, K, out_dtype):
    x, w, b, r = data(M, N, K, torch.bfloat16, True, True, True, out_dtype)
    y = r.clone()
    X.linear(x, w, bias=b, act="silu", gated=True, residual=y, y=y)
    sync()
    compare(y, x, w, b, r, "silu", True)


def test_one_operand_used_twice():
    # x as its own weight, and as the residual: inputs may overlap each other
    x = torch.randn(128, 128, generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    y = X.linear(x, x, act="gelu_tanh", residual=x)
    sync()
    compare(y, x, x, None, x, "gelu_tanh", False)
