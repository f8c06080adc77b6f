"""Root-mean-square norm with the residual's addition, its 8-bit form and its
backward as plain float64 definitions.

    h = x + r,  y = h w / sqrt(mean h^2 + eps)
    8 bits: s = max(max |y|, 2^-100) / 448 over a row or 128 columns of it,
            q = y / s rounded to the nearest e4m3 value, ties to even
    backward, u = dy w, rho = 1 / sqrt(mean h^2 + eps):
            dx = rho u - h rho^3 mean(u h) + dh,   gw = sum over rows of dy h rho

e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities; exponent
15 with mantissa 7 is NaN, so that the largest value is 448.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import numpy as np


def _f64(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


def rmsnorm(X, w=None, residual=None, eps: float = 1e-6):
    """(Y, H), neither rounded."""
    h = _f64(X) if residual is None else _f64(X) + _f64(residual)
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return (y if w is None else y * _f64(w)), h


def e4m3_values() -> np.ndarray:
    """The 256 codes' values (NaN for 0x7F and 0xFF)."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e.astype(np.float64) - 10))
    v = np.where((e == 15) & (m == 7), np.nan, v)
    return np.where(code >> 7, -v, v)


def round_e4m3(v) -> np.ndarray:
    """Nearest e4m3 value, ties to the even mantissa; |v| <= 464 (448 after rounding)."""
    v = _f64(v)
    pos = e4m3_values()[:127]  # ascending, 0 .. 448
    a = np.abs(v)
    i = np.clip(np.searchsorted(pos, a, side="right") - 1, 0, 126)
    j = np.minimum(i + 1, 126)
    lo, hi = a - pos[i], pos[j] - a
    pick = np.where((hi < lo) | ((hi == lo) & (i % 2 == 1)), j, i)
    out = np.where(np.isnan(v), np.nan, pos[pick])
    return np.copysign(out, v)


def scales(Y, group: int = 0) -> np.ndarray:
    """The scales of the rows (N x 1) or of each `group` columns of them."""
    Y = _f64(Y)
    d = Y.shape[1]
    cuts = list(range(0, d, group or d)) + [d]
    s = np.stack([np.abs(Y[:, i:j]).max(1) for i, j in zip(cuts, cuts[1:])], 1)
    return np.maximum(s, 2.0 ** -100) / 448.0


def spread(S, d: int, group: int = 0) -> np.ndarray:
    """Each column's scale (N x d)."""
    return np.repeat(S, group or d, axis=1)[:, :d]


def rmsnorm_backward(H, dY, w=None, dH=None, eps: float = 1e-6):
    """(dX, gw), neither rounded."""
    h, dy = _f64(H), _f64(dY)
    rho = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    u = dy if w is None else dy * _f64(w)
    dx = rho * u - h * rho ** 3 * (u * h).mean(1, keepdims=True)
    return (dx if dH is None else dx + _f64(dH)), (dy * h * rho).sum(0)
