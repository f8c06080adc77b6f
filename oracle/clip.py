"""Global gradient norm and clipping as plain float64 definitions.

    sumsq = sum of g^2 over every element of every tensor
    g <- g f,  f = 1 where sqrt(sumsq) <= max_norm, else max_norm / sqrt(sumsq)

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import math

import numpy as np


def sumsq(grads) -> float:
    return math.fsum(float(np.sum(np.asarray(g, np.float64) ** 2)) for g in grads)


def clip(grads, total: float, max_norm: float):
    """(norm, the scaled gradients)."""
    norm = math.sqrt(total) if total == total else math.nan
    f = 1.0 if norm <= max_norm else max_norm / norm
    return norm, [np.asarray(g, np.float64) * f for g in grads]
