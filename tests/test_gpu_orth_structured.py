"""Orthogonalised updates of matrices whose roundings do not average out: equal or few distinct
values, few rows that are not zero, low rank; at five steps and at the most that are admitted.

Tolerance.  X, A and Q are held to 2^-22.  Relative to the result's norm (|X_0| = 1, and the result's
is 0.68 or more) a rounding of X_k adds at most 2^-22 / 0.68 of |X_k|, which a direction that B lacks
carries on 3.4445 times a step and others less: 2^-22 * 3.4445^steps * (1 + 1 / 3.4445 + ...) / 0.68
< 2.1 * 2^-22 * 3.4445^steps, and A's and Q's, which X is multiplied with, as much again: 5 in all.
bf16 results are off by their own rounding besides, which is taken from the reference itself: where a
value lies so near to the middle of two bf16 numbers that the error above decides, either is as far off.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import orth as orc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _matrix(kind):
    g = torch.Generator().manual_seed(3)
    if kind.startswith("ones"):
        return torch.ones(*map(int, kind[4:].split("x")))
    if kind == "one-hot rows":
        m = torch.zeros(512, 512)
        m[torch.arange(32), torch.arange(32) * 7] = 1.0
        return m
    if kind == "identity":
        return torch.eye(256)
    if kind == "blocks":
        return torch.block_diag(*[torch.ones(32, 32)] * 8)
    m = torch.zeros(305, 700)
    if kind == "five rows":
        m[:5] = torch.randn(5, 700, generator=g)
        return m
    if kind == "five alike":
        m[:5] = 1.0 + 0.01 * torch.randn(5, 700, generator=g)
        return m
    if kind == "signs":
        return torch.sign(torch.randn(256, 256, generator=g))
    if kind == "rank 4":
        return torch.randn(640, 4, generator=g) @ torch.randn(4, 512, generator=g)
    return torch.randn(512, 512, generator=g)


KINDS = ["ones256x256", "ones1024x1024", "ones300x700", "ones700x300", "one-hot rows", "identity", "blocks",
         "five rows", "five alike", "signs", "rank 4", "gaussian"]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
def test_results_are_exact_to_their_rounding(dtype, kind):
    log(f"[orthogonalize, structured] {dtype} {kind}")
    a = _matrix(kind).to(DT[dtype]).cuda()
    for steps in (1, 5, 8):
        ref = orc.orthogonalize(host(a), steps)
        norm = np.linalg.norm(ref)
        own = np.linalg.norm(torch.from_numpy(ref).to(DT[dtype]).double().numpy() - ref) / norm
        tol = own + 5 * 2.0 ** -22 * 3.4445 ** steps
        off = np.linalg.norm(host(sn.sn_orthogonalize(a, steps=steps)) - ref) / norm
        log(f"  {steps} steps: {off:.2e} of the norm, its rounding {own:.2e}, at most {tol:.2e}")
        assert off <= tol


@pytest.mark.parametrize("steps", [5, 8])
def test_updates_stay_in_the_subspace(steps):
    """Gradients whose columns lie in 24 of 256 dimensions: what the update leaves outside is the bound
    above, and the rounding of W and G to float32, 2^-24, which grows alike."""
    log(f"[muon step, subspace] {steps} steps")
    r, k, c = 256, 24, 600
    g = torch.Generator().manual_seed(1)
    Q = torch.linalg.qr(torch.randn(r, k, dtype=torch.float64, generator=g))[0]
    W, G = ((Q @ torch.randn(k, c, dtype=torch.float64, generator=g)).float().cuda() for _ in range(2))
    w0 = host(W)
    sn.sn_muon_step(W, G, torch.zeros(r, c, device="cuda"), 0.1, steps=steps)
    step, q = host(W) - w0, Q.numpy()
    outside, norm = np.linalg.norm(step - q @ (q.T @ step)), np.linalg.norm(step)
    most = (5 * 2.0 ** -22 + 2 * 2.0 ** -24) * 3.4445 ** steps * norm + 2 * 2.0 ** -24 * np.linalg.norm(w0)
    log(f"  {outside:.3g} outside, at most {most:.3g}; the step {norm:.3g}")
    assert outside <= most and norm > 0.1
