"""The gated feed-forward block and its backward as plain float64 definitions.

    G = X Wg,  U = X Wu,  H = act(G) U
    dG = dH U act'(G),  dU = dH act(G),  dX = dG Wg^T + dU Wu^T,  gW = X^T dG, X^T dU

act: silu g / (1 + e^-g), gelu g (1 + erf(g / sqrt 2)) / 2, relu max(g, 0) (act'(0) = 0).

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import math

import numpy as np

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _f64(a):
    return np.asarray(a, dtype=np.float64)


def act(name: str, g):
    """(act(g), act'(g))."""
    g = _f64(g)
    if name == "relu":
        return np.maximum(g, 0.0), (g > 0).astype(np.float64)
    if name == "silu":
        e = np.exp(-np.abs(g))
        p = np.where(g >= 0, 1.0, e) / (1.0 + e)
        return g * p, p * (1.0 + g * (1.0 - p))
    p = 0.5 * _erfc(-g / math.sqrt(2.0))
    return g * p, p + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def gated_ff(X, Wg, Wu, name: str = "silu"):
    """(H, G, U), none rounded."""
    G, U = _f64(X) @ _f64(Wg), _f64(X) @ _f64(Wu)
    return act(name, G)[0] * U, G, U


def projections_backward(G, U, dH, name: str = "silu"):
    """(dG, dU)."""
    a, slope = act(name, G)
    return _f64(dH) * _f64(U) * slope, _f64(dH) * a


def products_backward(X, Wg, Wu, dG, dU):
    """(dX, gWg, gWu) from the projections' gradients."""
    X, dG, dU = _f64(X), _f64(dG), _f64(dU)
    return dG @ _f64(Wg).T + dU @ _f64(Wu).T, X.T @ dG, X.T @ dU
