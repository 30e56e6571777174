"""exfold_route_experts against its float64 definition: ids equal (both sides compare float64 values of
the same float32 or bf16 logits), weights within one float32 rounding."""

import numpy as np
import pytest
import torch

from oracle import operators_oracle as P
from paper_2608_24938_amd import exfold as X

from .gpu_common import DEV, sync

pytestmark = pytest.mark.gpu

# evaluated in float64 (relative error below 2^-40 for every input here) and rounded once to
# float32: half a step, 2^-24 of the value, and half the smallest subnormal below it
RTOL, ATOL = 2.0 ** -24 * (1 + 2.0 ** -10), 2.0 ** -149


def make(T, N, dtype, seed, kind):
    g = torch.Generator().manual_seed(seed)
    l = 1.5 * torch.randn(T, N, generator=g)
    if kind == "ties":
        l = torch.round(l)
    elif kind == "masked":
        l[torch.rand(T, N, generator=g) < 0.5] = -float("inf")
        l[::3] = -float("inf")
        l[1::5, 0] = float("nan")
        l[2::7] = torch.finfo(torch.float32).min
    elif kind == "wide":                      # scores that underflow or saturate
        l = l * 60
        l[::4, 0] = float("inf")
        l[1::6, ::2] = torch.finfo(torch.float32).max
    return l.to(dtype)


def check(logits, K, **kw):
    bias = kw.get("select_bias")
    ids, w = X.route_experts(logits, K, **kw)
    sync()
    ref = dict(kw, select_bias=None if bias is None else bias.cpu().numpy())
    rid, rw = P.route_experts(logits.float().cpu().numpy(), K, **ref)
    np.testing.assert_array_equal(ids.cpu().numpy(), rid)
    np.testing.assert_allclose(w.cpu().numpy().astype(np.float64), rw, rtol=RTOL, atol=ATOL)


SHAPES = [(1, 1, 1, 1, 1), (1, 8, 2, 1, 1), (3, 5, 5, 5, 5), (65, 64, 8, 8, 2), (33, 128, 8, 8, 4), (257, 128, 16, 1, 1),
          (40, 256, 16, 16, 1), (70, 160, 6, 8, 3), (19, 255, 7, 3, 2), (300, 60, 6, 6, 2), (17, 96, 4, 48, 2),
          (12, 256, 8, 256, 8), (129, 17, 3, 1, 1)]


@pytest.mark.parametrize("T,N,K,groups,keep", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("kind", ["plain", "ties", "masked", "wide"])
def test_routes(T, N, K, groups, keep, score, biased, kind):
    for dtype in (torch.float32, torch.bfloat16):
        for top2, renorm, scale in ((False, True, 1.0), (True, False, 2.5)):
            logits = make(T, N, dtype, T + N, kind).to(DEV)
            bias = None
            if biased:
                bias = 0.2 * torch.randn(N, generator=torch.Generator().manual_seed(N))
                if kind == "ties":
                    bias = torch.round(8 * bias) / 8
                bias = bias.to(DEV)
            check(logits, K, score=score, select_bias=bias, groups=groups, keep_groups=keep, group_top2=top2,
                  renorm=renorm, scale=scale)


def test_bias_that_masks_or_forces():
    logits = make(50, 24, torch.float32, 3, "masked").to(DEV)
    bias = torch.zeros(24)
    bias[3], bias[4], bias[5] = float("-inf"), float("nan"), float("inf")
    for score in ("softmax", "sigmoid"):
        for top2 in (False, True):
            check(logits, 4, score=score, select_bias=bias.to(DEV), groups=6, keep_groups=2, group_top2=top2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tokens_in_a_wider_buffer(dtype):
    # 5000 tokens: whole and partial workgroups of every build; rows 131 apart, the base 3 elements in
    buf = make(5000, 131 + 3, dtype, 11, "ties").to(DEV)
    before = buf.clone()
    logits = buf[:, 3:131]
    ids = torch.full((5002, 8), -7, dtype=torch.int32, device=DEV)
    w = torch.full((5002, 8), -7.0, device=DEV)
    bias = (0.1 * torch.randn(128, generator=torch.Generator().manual_seed(1))).to(DEV)
    kw = dict(score="sigmoid", select_bias=bias, groups=8, keep_groups=4, group_top2=True)
    X.route_experts(logits, 8, topk_ids=ids[1:5001], topk_w=w[1:5001], **kw)
    sync()
    rid, rw = P.route_experts(logits.float().cpu().numpy(), 8, **dict(kw, select_bias=bias.cpu().numpy()))
    np.testing.assert_array_equal(ids[1:5001].cpu().numpy(), rid)
    np.testing.assert_allclose(w[1:5001].cpu().numpy().astype(np.float64), rw, rtol=RTOL, atol=ATOL)
    assert (ids[[0, -1]] == -7).all() and (w[[0, -1]] == -7).all()          # rows beside the tokens' stay
    assert torch.equal(buf.view(torch.uint8), before.view(torch.uint8))


@pytest.mark.parametrize("T", [1, 64, 1000, 9000, 70000])
def test_batch_size_does_not_change_a_route(T):
    # every build routes a token alike: the first rows of a large batch against the same rows alone
    g = torch.Generator(device=DEV).manual_seed(T)
    logits = torch.randn(T, 200, generator=g, device=DEV).bfloat16()
    bias = 0.05 * torch.randn(200, generator=g, device=DEV)
    for kw in (dict(), dict(score="sigmoid", select_bias=bias, groups=8, keep_groups=3, group_top2=True)):
        ids, w = X.route_experts(logits, 8, **kw)
        for part in (1, 40):
            i2, w2 = X.route_experts(logits[-part:], 8, **kw)
            sync()
            n = min(part, T)
            assert torch.equal(ids[-n:], i2) and torch.equal(w[-n:], w2)
        again = X.route_experts(logits, 8, **kw)
        assert torch.equal(again[0], ids) and torch.equal(again[1], w)


def test_empty_batch_and_other_stream():
    ids, w = X.route_experts(torch.empty(0, 16, device=DEV), 4)
    assert ids.shape == (0, 4) and w.shape == (0, 4)
    side = torch.cuda.Stream()
    logits = make(100, 64, torch.float32, 5, "plain").to(DEV)
    sync()
    ids, w = X.route_experts(logits, 6, stream=side)
    side.synchronize()
    rid, _ = P.route_experts(logits.cpu().numpy(), 6)
    np.testing.assert_array_equal(ids.cpu().numpy(), rid)


def test_binding_refusals():
    l = torch.zeros(4, 8, device=DEV)
    for bad in (dict(score="other"), dict(select_bias=torch.zeros(7, device=DEV)), dict(select_bias=torch.zeros(8)),
                dict(topk_ids=torch.zeros(4, 3, dtype=torch.int32, device=DEV)),
                dict(topk_w=torch.zeros(4, 2, dtype=torch.float64, device=DEV))):
        with pytest.raises(ValueError):
            X.route_experts(l, 2, **bad)
    for bad in (l.t(), l.half(), l[0], l.expand(2, 4, 8)):
        with pytest.raises(ValueError):
            X.route_experts(bad, 2)
    with pytest.raises(X.ExfoldError):
        X.route_experts(l, 9)
    with pytest.raises(X.ExfoldError):
        X.route_experts(torch.zeros(1, 8, device=DEV).expand(4, 8), 2)      # rows on one another


def test_row_offsets_past_32_bits():
    T, N, ld = 70000, 96, 33000
    buf = torch.empty(T * ld, dtype=torch.bfloat16, device=DEV).view(T, ld)
    logits = buf[:, 8:8 + N]
    logits.copy_(torch.randn(T, N, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV))
    kw = dict(score="sigmoid", groups=6, keep_groups=3, group_top2=True)
    ids, w = X.route_experts(logits, 5, **kw)
    sync()
    for rows in (slice(0, 40), slice(T - 40, T)):
        rid, rw = P.route_experts(logits[rows].float().cpu().numpy(), 5, **kw)
        np.testing.assert_array_equal(ids[rows].cpu().numpy(), rid)
        np.testing.assert_allclose(w[rows].cpu().numpy().astype(np.float64), rw, rtol=RTOL, atol=ATOL)


@pytest.mark.parametrize("T", [1, 500])
def test_graph_replays_match_eager(T):
    kw = dict(score="sigmoid", groups=8, keep_groups=4, group_top2=True, scale=2.5,
              select_bias=(0.1 * torch.randn(128, generator=torch.Generator().manual_seed(1))).to(DEV))
    logits = make(T, 128, torch.float32, 1, "plain").to(DEV)
    ids = torch.empty(T, 8, dtype=torch.int32, device=DEV)
    w = torch.empty(T, 8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        X.route_experts(logits, 8, topk_ids=ids, topk_w=w, **kw)
    torch.cuda.current_stream().wait_stream(side)
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        X.route_experts(logits, 8, topk_ids=ids, topk_w=w, **kw)
    for rep in range(4):
        logits.copy_(make(T, 128, torch.float32, 10 + rep, "ties" if rep % 2 else "masked"))
        ref = X.route_experts(logits, 8, **kw)
        ids.fill_(-1)
        w.fill_(-1.0)
        graph.replay()
        sync()
        assert torch.equal(ids, ref[0]) and torch.equal(w, ref[1]), f"replay {rep}"
