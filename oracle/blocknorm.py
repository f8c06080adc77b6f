"""The end of a block and the start of the next, and its backward, as plain float64
definitions.

    z = x w_post / sqrt(mean x^2 + eps)  (post)  or  z = x
    h = alpha r + g z,   y = h w / sqrt(mean h^2 + eps),   g the gate or its sigmoid
    backward, n = h rho, u = dy w, q = 1 / sqrt(mean x^2 + eps), m = x q:
        dh = rho u - h rho^3 mean(u h) + dH,   dr = alpha dh,   dg = dh z g'
        v = g dh w_post,   dx = q v - x q^3 mean(v x)  (post)  or  dx = g dh
        gw = sum dy n,   gw_post = sum g dh m,   both over rows

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import numpy as np


def _f64(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


def gate_values(gate, fn: str):
    """(g, g') of a gate, 1 and 0 without one."""
    if gate is None:
        return np.float64(1.0), np.float64(0.0)
    g = _f64(gate)
    if fn == "none":
        return g, np.ones_like(g)
    g = np.where(g >= 0, 1.0 / (1.0 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1.0 + np.exp(-np.abs(g))))
    return g, g * (1.0 - g)


def _inv(h, eps):
    return 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)


def _z(X, w_post, post, eps):
    x = _f64(X)
    if not post:
        return x
    return x * _inv(x, eps) * (1.0 if w_post is None else _f64(w_post))


def block_norm(X, R, w=None, w_post=None, post=True, gate=None, fn="none", alpha=1.0, eps=1e-6):
    """(Y, H), neither rounded."""
    g, _ = gate_values(gate, fn)
    h = alpha * _f64(R) + g * _z(X, w_post, post, eps)
    return h * _inv(h, eps) * (1.0 if w is None else _f64(w)), h


def block_norm_backward(X, H, dY=None, w=None, w_post=None, post=True, gate=None, fn="none", alpha=1.0,
                        dH=None, eps=1e-6):
    """A dict of dX, dR, dgate (each token's), gw and gw_post, and of dh; none rounded."""
    x, h = _f64(X), _f64(H)
    dh, gw = np.zeros_like(x), np.zeros(x.shape[1])
    if dY is not None:
        rho = _inv(h, eps)
        u = _f64(dY) * (1.0 if w is None else _f64(w))
        dh = rho * u - h * rho ** 3 * (u * h).mean(1, keepdims=True)
        gw = (_f64(dY) * h * rho).sum(0)
    if dH is not None:
        dh = dh + _f64(dH)
    g, slope = gate_values(gate, fn)
    dz = dh * g
    out = {"dh": dh, "dR": alpha * dh, "gw": gw, "dgate": dh * _z(X, w_post, post, eps) * slope,
           "dX": dz, "gw_post": np.zeros(x.shape[1])}
    if post:
        q = _inv(x, eps)
        v = dz * (1.0 if w_post is None else _f64(w_post))
        out["gw_post"] = (dz * x * q).sum(0)
        out["dX"] = q * v - x * q ** 3 * (v * x).mean(1, keepdims=True)
    return out
