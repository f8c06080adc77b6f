"""Matrices of more than 2^31 elements: the last rows are right, and zeros stay zeros.  Tolerances are
those of the tests of each operator; rows and terms of zeros add nothing to an error."""
from __future__ import annotations

import pytest
import torch

import paper_2506_01260_amd as sn
import test_gpu_blocknorm as bn
import test_gpu_gated_ff as ff
import test_gpu_orth as orth
from gpu_helpers import host, log

pytestmark = pytest.mark.gpu

LAST = 40


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def _end(n, d, seed, dtype="bf16", std=1.0):
    """n x d, zero but for the last rows."""
    t = torch.zeros(n, d, dtype=bn.DT[dtype], device="cuda")
    t[n - LAST:] = bn._mat(seed, LAST, d, dtype, 0, std)
    return t


def test_block_norm():
    n, d = 270000, 8192
    assert n * d > 1 << 31
    log("[block norm, 2^31 elements]")
    X, R, dY = (_end(n, d, k) for k in (1, 2, 3))
    w, w1, gate = (bn._gain(k, d, "bf16") for k in (4, 5, 6))
    kw = dict(w_post=w1, gate=gate, gate_fn="sigmoid", alpha=0.5)
    Y, H = sn.sn_block_norm(X, R, w, **kw)
    tail = slice(n - LAST, n)
    bn._check_forward(Y[tail], H[tail], X[tail], R[tail], w, w1, True, gate, "sigmoid", 0.5, "bf16", "last rows")
    assert not bool(Y[:n - LAST].any()) and not bool(H[:n - LAST].any())
    sums = [torch.zeros(d, device="cuda") for _ in range(3)]
    dX, dR, _ = sn.sn_block_norm_backward(X, H, dY, w, gw=sums[0], gw_post=sums[1], dgate=sums[2], **kw)
    bn._check_backward((dX[tail], dR[tail], sums[2], *sums[:2]), 0.0, X[tail], H[tail], dY[tail], w, w1, True,
                       gate, "sigmoid", 0.5, None, "bf16", "last rows")
    assert not bool(dX[:n - LAST].any()) and not bool(dR[:n - LAST].any())


@pytest.mark.parametrize("width", [14336, 14331])
def test_gated_ff(width):
    n, d = 160000, 64
    assert n * width > 1 << 31
    log(f"[gated ff, 2^31 elements] {width}")
    X = _end(n, d, 1)
    Wg, Wu = (bn._mat(k, d, width, "bf16", 0, d ** -0.5) for k in (2, 3))
    H, G, U = sn.sn_gated_ff(X, Wg, Wu, save=True)
    tail = slice(n - LAST, n)
    ff._check_forward(H[tail], G[tail], U[tail], X[tail], Wg, Wu, "silu", "bf16", "last rows")
    assert not bool(H[:n - LAST].any()) and not bool(U[:n - LAST].any())
    dH = H
    dH[tail] = bn._mat(4, LAST, width, "bf16", 0, 0.1)
    dG, dU = torch.empty_like(G), torch.empty_like(U)
    dX, gWg, gWu = sn.sn_gated_ff_backward(X, Wg, Wu, G, U, dH, dG=dG, dU=dU)
    ff._check_backward(dX[tail], gWg, gWu, dG[tail], dU[tail], X[tail], Wg, Wu, G[tail], U[tail], dH[tail],
                       "silu", "bf16", "last rows")
    assert not bool(dX[:n - LAST].any()) and not bool(dG[:n - LAST].any()) and not bool(dU[:n - LAST].any())


def test_orthogonalize():
    r, c, h, w = 1 << 20, 2100, 60, 50
    assert r * c > 1 << 31
    log("[orthogonalize, 2^31 elements]")
    block = bn._mat(1, h, w, "f32")
    M = torch.zeros(r, c, device="cuda")
    M[r - h:, c - w:] = block
    got = sn.sn_orthogonalize(M)
    ref = orth.orc.orthogonalize(host(block))
    orth._near(host(got[r - h:, c - w:]), ref, orth._bound(host(block), 5, "f32"), "f32", "last rows")
    assert not bool(got[:r - h].any()) and not bool(got[r - h:, :c - w].any())
