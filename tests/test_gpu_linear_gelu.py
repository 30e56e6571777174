"""The gelu of bf16 outputs holds float32's bits of z Phi(z): where the residual takes the leading bits away, what is
left shows them.

z = x w is exact (two bf16 factors).  Half steps of float32 (2^-24 of the value) that z Phi(z) may be off by:
  the argument t = 1 / (1 + a m) of the polynomial: a rounding, and the reciprocal's full step of two: 3, times the
  slope d ln / d ln t of half the scaled complementary error function, at most 2.26: 6.8
  the polynomial: its fit 1.5; its steps one each, of which all but the last are damped by t and the ratio of the
  partial sum to the whole, in sum at most 2.2 (the magnitudes of its terms sum to 2.14 of it): 3.7
  the exponential's full step 2, two products 2, the sum with max(z, 0) 1: 5
  the exponent, h = c m m: two roundings and c's own 0.1, times ln 2 |h| = m^2 / 2: 1.1 m^2
together 17 + 1.1 z^2.  Adding r is one more of what is left, the output half a bf16 step of that."""

import numpy as np
import pytest
import torch
from scipy.special import log_ndtr

from paper_2608_24938_amd import exfold as X

from .gpu_common import DEV, sync

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24


@pytest.mark.parametrize("lo,hi", [(0.01, 1.0), (1.0, 3.0), (3.0, 7.0), (7.0, 12.0)])
@pytest.mark.parametrize("sign", [-1, 1])
def test_bits_below_the_residual(lo, hi, sign):
    g = torch.Generator().manual_seed(int(hi))
    x = (lo + (hi - lo) * torch.rand(2000, 1, generator=g)).bfloat16()
    w = (sign * (0.7 + 0.3 * torch.rand(500, 1, generator=g))).bfloat16()
    z = x.double().numpy() @ w.double().numpy().T
    exact = z * np.exp(log_ndtr(z))
    r = torch.from_numpy(-exact).bfloat16()
    left = exact + r.double().numpy()
    y = X.linear(x.to(DEV), w.to(DEV), act="gelu", residual=r.to(DEV))
    sync()
    err = np.abs(y.double().cpu().numpy() - left)
    lim = (17 + 1.1 * z * z) * U32 * np.abs(exact) + (2.0 ** -8 + U32) * np.abs(left) + 2.0 ** -126
    fine = np.abs(left) < 2.0 ** -13 * np.abs(exact)                 # the output's own half step is below 2^-21 here
    assert fine.sum() > 20000
    over = ((err - lim) / np.abs(exact))[fine]
    assert (err <= lim)[fine].all(), f"{over.max() / U32} half steps too many, at z = {z[fine][over.argmax()]}"


def test_far_values_and_infinities():
    x = torch.tensor([[20.0], [-20.0], [3e38], [-3e38], [float("inf")], [float("nan")], [0.0]], dtype=torch.bfloat16, device=DEV)
    y = X.linear(x, torch.ones(40, 1, dtype=torch.bfloat16, device=DEV), act="gelu")
    sync()
    assert (y[0] == 20).all() and (y[1] == 0).all() and (y[2] == x[2]).all() and (y[3] == 0).all()
    assert (y[4] == float("inf")).all() and y[5].isnan().all() and (y[6] == 0).all()
