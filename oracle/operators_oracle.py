"""float64 NumPy definitions of the routing and matrix-product operators (exfold_route_experts,
exfold_linear_forward): test infrastructure that shares no code with the library."""

from __future__ import annotations

import numpy as np
from scipy.special import ndtr


def scores(logits, score):
    """[T, N] float64 scores; 0 where the logit is -inf or NaN (masked); +inf counts as the largest float32."""
    l = np.array(logits, dtype=np.float64)
    masked = ~(l > -np.inf)
    l = np.minimum(np.where(masked, -np.inf, l), np.finfo(np.float32).max)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        if score == "softmax":
            top = l.max(axis=1, keepdims=True)
            e = np.where(masked, 0.0, np.exp(l - np.where(np.isneginf(top), 0.0, top)))
            p = e / np.where(top > -np.inf, e.sum(axis=1, keepdims=True), 1.0)
        else:
            p = np.where(masked, 0.0, 1.0 / (1.0 + np.exp(-l)))
    return l, p, masked


def route_experts(logits, k, score="softmax", select_bias=None, groups=1, keep_groups=1, group_top2=False,
                  renorm=True, scale=1.0):
    """(ids [T, k] int32, weights [T, k] float64), token by token from the definition."""
    l, p, masked = scores(logits, score)
    T, N = l.shape
    b = np.zeros(N) if select_bias is None else np.asarray(select_bias, dtype=np.float64)
    size = N // groups
    ids = np.empty((T, k), dtype=np.int32)
    w = np.empty((T, k))
    for t in range(T):
        s = p[t] + b
        dead = masked[t] | ~(s > -np.inf)
        v = np.where(dead, -np.inf, l[t] if select_bias is None else s)
        cand = range(N)
        if groups > 1:
            value = []
            for g in range(groups):
                inside = [e for e in range(g * size, (g + 1) * size) if not dead[e]]
                if not inside:
                    value.append(-np.inf)
                elif group_top2:
                    value.append(sum(sorted((s[e] for e in inside), reverse=True)[:2]))
                else:
                    value.append(max(v[e] for e in inside))
            kept = sorted(range(groups), key=lambda g: (-value[g], g))[:keep_groups]
            cand = [e for g in sorted(kept) for e in range(g * size, (g + 1) * size)]
        pick = sorted(cand, key=lambda e: (-v[e], e))[:k]
        pw = np.array([0.0 if dead[e] else p[t, e] for e in pick])
        if renorm:
            pw = pw / pw.sum() if pw.sum() > 0 else np.zeros(k)
        ids[t] = pick
        w[t] = pw * np.float64(np.float32(scale))
    return ids, w


def activate(act, z):
    if act == "relu":
        return np.maximum(z, 0.0)
    if act == "silu":
        return z * 0.5 * (1.0 + np.tanh(0.5 * z))
    if act == "gelu":
        return z * ndtr(z)
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (z + 0.044715 * z ** 3)))
    assert act == "none"
    return z


def linear(x, w, bias=None, act="none", gated=False, residual=None):
    """(y float64, mag): mag bounds |term| sums for error bounds: sum |x w| + |b| of the gate and the up product."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    z, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        z, mag = z + np.asarray(bias, np.float64), mag + np.abs(np.asarray(bias, np.float64))
    if gated:
        n = w.shape[0] // 2
        y = activate(act, z[:, :n]) * z[:, n:]
    else:
        y = activate(act, z)
    return (y if residual is None else y + np.asarray(residual, np.float64)), z, mag
