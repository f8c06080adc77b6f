"""Orthogonalised updates as plain float64 definitions.

    X = B / |B|_F, then steps times X <- (a I + b A + c A^2) X with A = X X^T
    M <- mu M + G,  B = G + mu M or M,  W <- W - lr scale X - decay W

The polynomial acts on the singular values alone: by_singular_values() applies it to them,
f(s) = a s + b s^3 + c s^5.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import numpy as np

A, B, C = 3.4445, -4.7750, 2.0315


def f(s, steps: int = 1):
    """The steps' polynomial of singular values."""
    s = np.asarray(s, dtype=np.float64)
    for _ in range(steps):
        s = A * s + B * s ** 3 + C * s ** 5
    return s


def iterates(M, steps: int = 5):
    """[X_0, ..., X_steps]; the shorter side first inside, as the definition's X X^T."""
    x = np.asarray(M, dtype=np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    n = np.linalg.norm(x)
    x = x / n if n > 0 else x
    out = [x]
    for _ in range(steps):
        p = x @ x.T
        x = A * x + (B * p + C * (p @ p)) @ x
        out.append(x)
    return [v.T if tall else v for v in out]


def orthogonalize(M, steps: int = 5):
    return iterates(M, steps)[-1]


def by_singular_values(M, steps: int = 5):
    u, s, v = np.linalg.svd(np.asarray(M, dtype=np.float64), full_matrices=False)
    n = np.sqrt((s * s).sum())
    return (u * f(s / n if n > 0 else s, steps)) @ v


def momentum(M, G, mu: float, nesterov: bool = True):
    """(new momentum, matrix to orthogonalise)."""
    m = mu * np.asarray(M, dtype=np.float64) + np.asarray(G, dtype=np.float64)
    return m, np.asarray(G, dtype=np.float64) + mu * m if nesterov else m


def muon_step(W, G, M, lr, mu=0.95, nesterov=True, decay=0.0, scale=1.0, steps=5):
    """(W, M) after the step, neither rounded."""
    m, b = momentum(M, G, mu, nesterov)
    return np.asarray(W, dtype=np.float64) * (1.0 - decay) - lr * scale * orthogonalize(b, steps), m
