"""Float64 CPU reference of the operators around the mixer (linear layer,
embedding), in plain NumPy: test infrastructure, no code shared with the HIP
path."""

from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def activate(y, act):
    if act == "relu":
        return np.maximum(y, 0.0)
    if act == "gelu":
        return 0.5 * y * (1.0 + _erf(y / math.sqrt(2.0)))
    if act == "silu":
        return y / (1.0 + np.exp(-y))
    return y


def slope(y, act):
    if act == "relu":
        return (y > 0).astype(np.float64)
    if act == "gelu":
        return 0.5 * (1.0 + _erf(y / math.sqrt(2.0))) + y * np.exp(-0.5 * y * y) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-y))
        return s + y * s * (1.0 - s)
    return np.ones_like(y)


def linear_forward(X, W, bias, residual, act):
    """(out, pre) of out = residual + act(X W + bias)."""
    pre = X @ W + (0.0 if bias is None else bias)
    return activate(pre, act) + (0.0 if residual is None else residual), pre


def linear_backward(X, W, pre, dOut, act):
    """dX, dW, dbias for dP = dOut * act'(pre)."""
    dP = dOut if act == "none" else dOut * slope(pre, act)
    return dP @ W.T, X.T @ dP, dP.sum(0)


def embedding_backward(ids, dOut, V, scale):
    out = np.zeros((V, dOut.shape[-1]))
    for t, v in enumerate(ids):
        if 0 <= v < V:
            out[v] += dOut[t]
    return scale * out
