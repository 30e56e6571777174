"""Routes of tokens with few or no live experts (padding, masks) through selection, the safeguarded fold and the
experts: weights of zero stay zero and nothing becomes NaN."""

import numpy as np
import pytest
import torch

from oracle import exfold_oracle as O
from oracle import operators_oracle as P
from paper_2608_24938_amd import exfold as X
from paper_2608_24938_amd import synth

from .gpu_common import DEV, LayerPair, sync, to_dev

pytestmark = pytest.mark.gpu

OPTS = [{}, dict(renorm=True), dict(confidence=True), dict(confidence=True, renorm=True),
        dict(loss_cap=0.7, confidence=True, renorm=True)]


def masked_logits(T, N, seed):
    g = torch.Generator().manual_seed(seed)
    l = 1.5 * torch.randn(T, N, generator=g)
    l[torch.rand(T, N, generator=g) < 0.4] = -float("inf")
    l[::3] = -float("inf")                                           # no live expert
    l[1::5, 1:] = -float("inf")                                      # at most one
    return l


@pytest.mark.parametrize("T,N,K,kp", [(1, 8, 2, 1), (65, 32, 6, 2), (200, 64, 8, 8), (90, 48, 12, 3), (33, 256, 16, 5)])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("opts", OPTS, ids=lambda o: "-".join(f"{k}={v}" for k, v in o.items()) or "plain")
def test_fold_of_masked_tokens(T, N, K, kp, renorm, opts):
    rng = np.random.default_rng(T + K)
    S = (rng.standard_normal((N, N)) * 1.5).astype(np.float32)
    L, h = (rng.random((N, N)) * 1.3).astype(np.float32), rng.random(N).astype(np.float32)
    ids, w = X.route_experts(masked_logits(T, N, K).to(DEV), K, score="sigmoid", renorm=renorm, scale=2.5)
    _, _, keep = X.select_prefill(to_dev(h), kp, topk_ids=ids, topk_w=w)
    out_ids, out_w = X.fold_gates("prefill", kp, ids, w, to_dev(S), to_dev(L), keep=keep, **opts)
    sync()
    wf, out = w.cpu().numpy(), out_w.cpu().numpy()
    assert (wf[::3] == 0).all()
    ri, rw = O.fold_prefill_safeguarded(ids.cpu().numpy(), wf, keep.cpu().numpy().astype(bool), S, L, **opts)
    np.testing.assert_array_equal(out_ids.cpu().numpy(), ri)
    assert np.isfinite(out).all() and (out[::3] == 0).all()
    np.testing.assert_array_equal(out.view(np.uint32), rw.view(np.uint32))


@pytest.mark.parametrize("phase,budget", [("prefill", 2), ("decode", 8)])
def test_padding_tokens_leave_the_layer_as_zeros(phase, budget):
    shape = synth.LayerShape("pad", d=256, inter=128, n_experts=32, top_k=4, dtype="bf16", router_bias=False)
    lp, T = LayerPair(shape, seed=3), 70
    S, L, h = (to_dev(a) for a in synth.synthetic_tables(32, seed=3))
    x = to_dev(synth.tokens(shape, T, seed=3))
    logits = X.linear(x, lp.dev.w_router, out_dtype=torch.float32)
    logits[10:20] = -float("inf")
    ids, w = X.route_experts(logits, 4)
    if phase == "prefill":
        _, _, keep = X.select_prefill(h, budget, topk_ids=ids, topk_w=w)
        oi, ow = X.fold_gates(phase, budget, ids, w, S, L, keep=keep, confidence=True, renorm=True)
    else:
        _, _, pool, size = X.select_decode_pool(h, budget, topk_ids=ids, topk_w=w)
        oi, ow = X.fold_gates(phase, budget, ids, w, S, L, pool=pool, pool_size=size)
    y = X.moe_execute(lp.dev, x, oi, ow)
    sync()
    rid, rw = P.route_experts(logits.cpu().numpy(), 4)
    np.testing.assert_array_equal(ids.cpu().numpy(), rid)
    assert (y[10:20] == 0).all() and y.isfinite().all()
    assert (y[:10] != 0).any(1).all() and (y[20:] != 0).any(1).all()
