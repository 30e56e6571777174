"""Refusals of exfold_route_experts and exfold_linear_forward: every one is decided on the host before
anything is enqueued, so the pointers here are never dereferenced (no GPU)."""

import ctypes

import pytest
import torch

from paper_2608_24938_amd import exfold as X

F = 0x100000   # far from each other: no buffer below overlaps another unless a test says so
LOGITS, BIAS, IDS, W = F, 16 * F, 32 * F, 48 * F


def route(T=4, N=8, K=2, ld=None, dtype=X.F32, logits=LOGITS, ids=IDS, w=W, routing=True, **kw):
    r = dict(score=0, group_value=0, n_groups=1, keep_groups=1, renorm=1, scale=1.0, select_bias=None)
    r.update(kw)
    rs = X._Routing(*r.values())
    return X.lib().exfold_route_experts(ctypes.byref(rs) if routing else None, logits, dtype, N if ld is None else ld,
                                        T, N, K, ids, w, None)


@pytest.mark.parametrize("kw,code", [
    (dict(routing=False), X.ERR_NULL), (dict(logits=None), X.ERR_NULL), (dict(ids=None), X.ERR_NULL),
    (dict(w=None), X.ERR_NULL),
    (dict(dtype=2), X.ERR_DTYPE),
    (dict(T=-1), X.ERR_SHAPE), (dict(N=0), X.ERR_SHAPE), (dict(K=0), X.ERR_SHAPE), (dict(K=9), X.ERR_SHAPE),
    (dict(T=(1 << 22) + 1), X.ERR_SHAPE), (dict(ld=7), X.ERR_SHAPE), (dict(ld=(1 << 31) + 1), X.ERR_SHAPE),
    (dict(N=257), X.ERR_UNSUPPORTED), (dict(N=64, K=17), X.ERR_UNSUPPORTED),
    (dict(score=2), X.ERR_ARG), (dict(score=-1), X.ERR_ARG), (dict(group_value=2), X.ERR_ARG),
    (dict(scale=0.0), X.ERR_ARG), (dict(scale=-1.0), X.ERR_ARG), (dict(scale=float("nan")), X.ERR_ARG),
    (dict(scale=float("inf")), X.ERR_ARG),
    (dict(n_groups=3), X.ERR_SHAPE), (dict(n_groups=0), X.ERR_SHAPE), (dict(n_groups=16), X.ERR_SHAPE),
    (dict(n_groups=4, keep_groups=0), X.ERR_SHAPE), (dict(n_groups=4, keep_groups=5), X.ERR_SHAPE),
    (dict(n_groups=8, keep_groups=1), X.ERR_SHAPE),                        # one expert for two routes
    (dict(logits=LOGITS + 2), X.ERR_ALIGN), (dict(ids=IDS + 1), X.ERR_ALIGN), (dict(w=W + 2), X.ERR_ALIGN),
    (dict(select_bias=BIAS + 1), X.ERR_ALIGN), (dict(dtype=X.BF16, logits=LOGITS + 1), X.ERR_ALIGN),
    (dict(ids=W), X.ERR_ARG), (dict(ids=LOGITS + 4 * 31), X.ERR_ARG), (dict(w=LOGITS), X.ERR_ARG),
    (dict(select_bias=W + 4 * 7), X.ERR_ARG),
])
def test_route_refusals(kw, code):
    assert route(**kw) == code


def test_route_no_tokens_is_a_no_op():
    assert route(T=0) == X.OK
    assert route(T=0, logits=None, ids=None, w=None) == X.OK
    assert route(T=0, K=9) == X.ERR_SHAPE


XP, WP, BP, RP, YP, WS = F, 64 * F, 128 * F, 192 * F, 256 * F, 320 * F


def linear(M=100, x=XP, ldx=None, res=None, ldr=0, y=YP, ldy=None, ws=WS, ws_bytes=None, lin=True, **kw):
    a = dict(n_in=4096, n_out=32, ldw=None, w=WP, bias=None, dtype=X.BF16, out_dtype=None, act=0, gated=0)
    a.update(kw)
    a["ldw"] = a["n_in"] if a["ldw"] is None else a["ldw"]
    a["out_dtype"] = a["dtype"] if a["out_dtype"] is None else a["out_dtype"]
    ls = X._Linear(*a.values())
    p = ctypes.byref(ls) if lin else None
    size = X.lib().exfold_linear_workspace_size(p, M)
    st = X.lib().exfold_linear_forward(p, x, a["n_in"] if ldx is None else ldx, M, res, ldr, y,
                                       a["n_out"] if ldy is None else ldy, ws, size if ws_bytes is None else ws_bytes,
                                       None)
    return st, size


@pytest.mark.parametrize("kw,code,sized", [
    (dict(lin=False), X.ERR_NULL, False), (dict(w=None), X.ERR_NULL, False),
    (dict(x=None), X.ERR_NULL, True), (dict(y=None), X.ERR_NULL, True), (dict(ws=None), X.ERR_NULL, True),
    (dict(dtype=2), X.ERR_DTYPE, False), (dict(dtype=X.F32, out_dtype=X.BF16), X.ERR_DTYPE, False),
    (dict(out_dtype=5), X.ERR_DTYPE, False),
    (dict(act=5), X.ERR_ARG, False), (dict(act=-1), X.ERR_ARG, False), (dict(gated=2), X.ERR_ARG, False),
    (dict(n_in=0), X.ERR_SHAPE, False), (dict(n_out=0), X.ERR_SHAPE, False), (dict(n_in=(1 << 17) + 1), X.ERR_SHAPE, False),
    (dict(n_out=(1 << 17) + 1), X.ERR_SHAPE, False), (dict(ldw=4095), X.ERR_SHAPE, False),
    (dict(ldw=(1 << 31) + 1), X.ERR_SHAPE, False), (dict(M=-1), X.ERR_SHAPE, False),
    (dict(M=(1 << 22) + 1), X.ERR_SHAPE, False), (dict(M=1 << 22, n_out=1 << 13), X.ERR_SHAPE, False),
    (dict(ldx=4095), X.ERR_SHAPE, True), (dict(ldy=31), X.ERR_SHAPE, True), (dict(res=RP, ldr=31), X.ERR_SHAPE, True),
    (dict(ldx=(1 << 31) + 1), X.ERR_SHAPE, True), (dict(ldy=(1 << 31) + 1), X.ERR_SHAPE, True),
    (dict(w=WP + 1), X.ERR_ALIGN, False), (dict(bias=BP + 2), X.ERR_ALIGN, False), (dict(x=XP + 1), X.ERR_ALIGN, True),
    (dict(y=YP + 1), X.ERR_ALIGN, True), (dict(out_dtype=X.F32, y=YP + 2), X.ERR_ALIGN, True),
    (dict(res=RP + 1, ldr=32), X.ERR_ALIGN, True),
    (dict(ws_bytes=0), X.ERR_WORKSPACE, True), (dict(ws=WS + 8), X.ERR_WORKSPACE, True),
    (dict(y=XP), X.ERR_ARG, True), (dict(y=WP + 2), X.ERR_ARG, True), (dict(y=BP + 4, bias=BP), X.ERR_ARG, True),
    (dict(y=YP, res=YP + 2, ldr=32), X.ERR_ARG, True), (dict(y=YP, res=YP, ldr=64), X.ERR_ARG, True),
    (dict(y=WS + 16), X.ERR_ARG, True), (dict(x=WS - 16), X.ERR_ARG, True),
    (dict(y=XP + 2 * 4090, ldx=4200, ldy=4200), X.ERR_ARG, True),         # from x's column 4090 on
])
def test_linear_refusals(kw, code, sized):
    st, size = linear(**kw)
    assert st == code
    assert (size > 0) == sized


def test_linear_needs_a_workspace_only_for_partial_sums():
    assert linear(x=None)[1] > 0                                          # 4096 long, one tile of outputs
    st, size = linear(n_in=64, x=None, ws=None)
    assert (st, size) == (X.ERR_NULL, 0)
    assert linear(n_in=64, n_out=1 << 15, x=None, ws=None)[1] == 0


def test_linear_no_rows_is_a_no_op():
    assert linear(M=0)[0] == X.OK
    assert linear(M=0, x=None, y=None, ws=None)[0] == X.OK
    assert linear(M=0, ldx=3)[0] == X.ERR_SHAPE


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(4, 8), torch.zeros(2, 8)
    with pytest.raises(ValueError, match="on the GPU"):
        X.linear(x, w)
    with pytest.raises(ValueError, match="on the GPU"):
        X.route_experts(torch.zeros(4, 8), 2)
