"""A sum that is no number stays none through every activation, on every kernel family and epilogue: a NaN in a
row of x, a NaN in a weight row (gated: of the gate), infinities of both signs in a row."""

import pytest
import torch

from .gpu_common import DEV, sync
from .linear_builds import build
from .test_gpu_linear import compare, data
from paper_2608_24938_amd import exfold as X

pytestmark = pytest.mark.gpu

PATHS = [(4, 40, 64, ("few", 4, 2, "pieces")), (5, 33, 45, ("few", 4, 2, "any")), (96, 130, 192, ("ring", 32, 64, "again")),
         (64, 130, 8192, ("ring", 32, 64, "again", "split")), (200, 90, 45, ("tile",)), (1190, 5230, 128, ("wide",))]


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K,path", PATHS)
def test_nan_goes_through(M, N, K, path, out_dtype, gated, act):
    n = N // 2 if gated else N
    assert build(M, n, K, gated=gated, x_aligned=K % 8 == 0) == path
    x, w, b, r = data(M, n, K, torch.bfloat16, gated, True, True, out_dtype)
    w[:, :2] = w[:, :2].abs() + 0.25
    x[0, K // 2] = float("nan")
    x[1, 0], x[1, 1] = float("inf"), float("-inf")
    w[n - 1, 3] = float("nan")                                      # gated: the last gate row
    y = X.linear(x, w, bias=b, act=act, gated=gated, residual=r, out_dtype=out_dtype)
    sync()
    assert y[:2].isnan().all() and y[:, n - 1].isnan().all()
    rows = [i for i in range(w.shape[0]) if i % n != n - 1]
    compare(y[2:, :n - 1], x[2:], w[rows], b[rows], r[2:, :n - 1], act, gated)


@pytest.mark.parametrize("M", [3, 40])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_float32_inputs_and_infinities_of_the_relu(M, dtype):
    x, w, _, _ = data(M, 48, 64, dtype, False, False, False, dtype)
    x[0, 5] = float("nan")
    x[1, 0] = float("inf")
    w[:, 0] = torch.where(torch.arange(48, device=DEV) % 2 == 0, 1.0, -1.0).to(dtype)
    y = X.linear(x, w, act="relu")
    sync()
    assert y[0].isnan().all()
    assert (y[1, ::2] == float("inf")).all() and (y[1, 1::2] == 0).all()
    compare(y[2:], x[2:], w, None, None, "relu", False)
