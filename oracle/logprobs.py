"""Token log probabilities, entropy, alternatives and their gradients as plain
float64 definitions.

For a row of logits z and scale c:

    p_j = exp(c z_j) / sum_k exp(c z_k)
    logp = log p_t for the given token t (0 where t = -1)
    H = -sum_j p_j log p_j            (0 log 0 = 0)
    alternatives: the largest logits in descending order, the lower id first
    among equals, with their log p
    d/dz_j (gl logp + gh H) = c (gl (d_jt - p_j) - gh p_j (log p_j + H))

A logit of -inf has p = 0 and log p = -inf.  A row whose logits are all -inf has
p = 0 throughout, logp -inf and H 0.  A row that holds NaN or +inf has no
distribution: NaN everywhere, and -1 for the alternatives' ids.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import numpy as np


def log_p(Z, scale: float = 1.0) -> np.ndarray:
    """log p of every logit (N x V, float64)."""
    a = scale * np.asarray(Z, dtype=np.float64)
    out = np.full(a.shape, np.nan)
    for i, row in enumerate(a):
        if np.isnan(row).any() or np.isposinf(row).any():
            continue
        if np.isneginf(row).all():
            out[i] = -np.inf
            continue
        top = row.max()
        out[i] = (row - top) - np.log(np.sum(np.exp(row - top)))
    return out


def _plogp(lp):
    p = np.exp(lp)
    return np.where(p > 0, p * np.where(p > 0, lp, 0.0), p)


def token_logprobs(Z, tok, n_top: int = 0, scale: float = 1.0):
    """(logp, entropy, stats, top_logp, top_id)."""
    Z = np.asarray(Z, dtype=np.float64)
    N, V = Z.shape
    lp = log_p(Z, scale)
    tok = np.asarray(tok)
    logp = np.where(tok >= 0, lp[np.arange(N), np.maximum(tok, 0)], 0.0)
    entropy = -_plogp(lp).sum(1)
    stats = np.empty((N, 2))
    top_logp, top_id = np.empty((N, n_top)), np.empty((N, n_top), dtype=np.int64)
    for i in range(N):
        if np.isnan(lp[i]).any():
            stats[i], top_logp[i], top_id[i], entropy[i] = np.nan, np.nan, -1, np.nan
            continue
        m = Z[i].max()
        stats[i, 0] = m
        at = int(np.argmax(Z[i]))
        stats[i, 1] = -np.inf if np.isneginf(m) else -lp[i, at]
        order = sorted(range(V), key=lambda j: (-Z[i, j], j))[:n_top]
        top_id[i], top_logp[i] = order, lp[i, order]
    return logp, entropy, stats, top_logp, top_id


def token_logprobs_backward(Z, tok, g_logp=None, g_entropy=None, scale: float = 1.0):
    """dZ for the gradients of logp and entropy.  A row that nothing flows into is 0."""
    lp = log_p(Z, scale)
    N, V = lp.shape
    tok = np.asarray(tok)
    gl = np.zeros(N) if g_logp is None else np.where(tok >= 0, np.asarray(g_logp, np.float64), 0.0)
    gh = np.zeros(N) if g_entropy is None else np.asarray(g_entropy, np.float64)
    p, plogp = np.exp(lp), _plogp(lp)
    H = -plogp.sum(1)
    hit = (np.arange(V)[None] == tok[:, None]).astype(np.float64)
    d = scale * (gl[:, None] * (hit - p) - gh[:, None] * (plogp + p * H[:, None]))
    d[(gl == 0) & (gh == 0)] = 0.0
    return d


def token_loss(Z, tok, weight=None, scale: float = 1.0):
    """(logp, dZ) of the loss -sum_i weight_i logp_i."""
    w = np.ones(len(tok)) if weight is None else np.asarray(weight, np.float64)
    logp = token_logprobs(Z, tok, 0, scale)[0]
    return logp, token_logprobs_backward(Z, tok, g_logp=-w, scale=scale)
