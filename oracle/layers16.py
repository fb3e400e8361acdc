"""Layers kept in 16 bits, in 64-bit numpy: the projection with its epilogue and linear attention with a decay per head.

Every function also returns what its result is made of in absolute values (all products and additions with their
signs removed): rounding errors of a sum are bounded by that, not by the sum.
"""
from __future__ import annotations

import math

import numpy as np

_ERF = np.vectorize(math.erf, otypes=[np.float64])


def activate(v, act):
    v = np.asarray(v, dtype=np.float64)
    with np.errstate(over="ignore"):
        if act == "relu":
            return np.maximum(v, 0.0)
        if act == "silu":
            return v / (1.0 + np.exp(-v))
        if act == "gelu":
            return 0.5 * v * (1.0 + _ERF(v / math.sqrt(2.0)))
        if act == "gelu_tanh":
            return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
        if act == "sigmoid":
            return 1.0 / (1.0 + np.exp(-v))
    assert act == "none", act
    return v


def linear(x, W, bias=None, residual=None, act="none"):
    """(out, sums of absolute products plus |bias|) of act(x W^T + bias) + residual; x [M, K], W [N, K]."""
    x, W = np.asarray(x, dtype=np.float64), np.asarray(W, dtype=np.float64)
    v, size = x @ W.T, np.abs(x) @ np.abs(W).T
    if bias is not None:
        v, size = v + bias, size + np.abs(bias)
    out = activate(v, act)
    return (out if residual is None else out + np.asarray(residual, dtype=np.float64)), size


def linattn(q, k, v, g=None, state=None, lens=None, scale=1.0):
    """Token by token.  q, k [B, L, Hk, dk], v [B, L, Hv, dv], g [B, L, Hv] or [Hv] or None, state [B, Hv, dk, dv] or None.

    Returns (out [B, L, Hv, dv] with NaN behind a sequence's end, state, and both in absolute values)."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    B, L, Hk, dk = q.shape
    Hv, dv = v.shape[2:]
    q, k = np.repeat(q, Hv // Hk, axis=2), np.repeat(k, Hv // Hk, axis=2)
    a = np.ones((B, L, Hv)) if g is None else np.broadcast_to(np.exp(np.minimum(np.asarray(g, dtype=np.float64), 0.0)), (B, L, Hv))
    S = np.zeros((B, Hv, dk, dv)) if state is None else np.array(state, dtype=np.float64)
    size = np.abs(S)
    out, out_size = np.full((B, L, Hv, dv), np.nan), np.full((B, L, Hv, dv), np.nan)
    for b in range(B):
        for t in range(L if lens is None else int(min(max(lens[b], 0), L))):
            S[b] = a[b, t][:, None, None] * S[b] + k[b, t][:, :, None] * v[b, t][:, None, :]
            size[b] = a[b, t][:, None, None] * size[b] + np.abs(k[b, t][:, :, None] * v[b, t][:, None, :])
            out[b, t] = scale * np.einsum("hd,hde->he", q[b, t], S[b])
            out_size[b, t] = abs(scale) * np.einsum("hd,hde->he", np.abs(q[b, t]), size[b])
    return out, S, out_size, size
