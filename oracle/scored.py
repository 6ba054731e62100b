"""Scored attention and its gradients from their definitions, in 64 bits (oracle side; test infrastructure).

One (batch, head) plane of tokens in natural order: scores are capped, biased and masked, the softmax is taken over what is
visible, a query that sees nothing has a zero row.
"""
import math

import numpy as np


def visible(keep, positions=None, limits=None, documents=None):
    """bool [N, N]: keep (from the tile lists), restricted by limits and documents."""
    seen = np.array(keep, dtype=bool)
    if limits is not None:
        seen &= positions[None, :] <= limits[:, None]
    if documents is not None:
        seen &= (documents[:, None] == documents[None, :]) & (documents[:, None] >= 0)
    return seen


def scores(q, k, scale, cap=0.0, slope=None, positions=None):
    """(scores, derivative of the capped scores) before the mask."""
    s = q @ k.T * scale
    steep = np.ones_like(s)
    if cap:
        steep = 1 / np.cosh(np.minimum(np.abs(s / cap), 300.0)) ** 2
        s = cap * np.tanh(s / cap)
    if slope is not None:
        s = s - slope * np.abs(positions[:, None] - positions[None, :])
    return s, steep


def forward(q, k, v, seen, scale, **how):
    """(out, lse, weights)"""
    s, _ = scores(q, k, scale, **how)
    s = np.where(seen, s, -math.inf)
    top = np.max(s, axis=1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    e = np.exp(s - top)
    total = e.sum(axis=1, keepdims=True)
    p = np.divide(e, total, out=np.zeros_like(e), where=total > 0)
    with np.errstate(divide="ignore"):
        lse = (np.log(total) + top)[:, 0]
    return p @ v, lse, p


def backward(dout, q, k, v, seen, scale, **how):
    """(dq, dk, dv, dS, weights)"""
    out, _, p = forward(q, k, v, seen, scale, **how)
    _, steep = scores(q, k, scale, **how)
    dp = dout @ v.T
    ds = p * (dp - (dout * out).sum(axis=1, keepdims=True)) * steep
    return scale * ds @ k, scale * ds.T @ q, p.T @ dout, ds, p
