"""Sigmoid gates far from 0, in both directions: the gate's and its derivative's relative error stays
what it is near 0, also where 1 - sigmoid is a small part of 1 and in the float32 sums of bf16 calls.
Tolerances are those of test_gpu_blocknorm (its derivation: a sigmoid 8 u, its derivative 16 u of itself)."""
from __future__ import annotations

import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from test_gpu_blocknorm import DT, EPS, _check_backward, _check_forward, _gain, _mat

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["row", "token"])
@pytest.mark.parametrize("n,d", [(5, 192), (9, 3), (300, 777), (3, 20000)], ids=str)
def test_far_gates(dtype, kind, n, d):
    log(f"[block norm, far gates] {dtype} {kind} {n} x {d}")
    X, R = _mat(1, n, d, dtype), _mat(2, n, d, dtype, 0, 2.0)
    dY, dH = _mat(3, n, d, dtype, 0, 0.1), _mat(4, n, d, dtype, 0, 0.1)
    w, w1 = _gain(5, d, dtype), _gain(6, d, dtype)
    count = d if kind == "row" else n * d
    # (up to 20: the oracle takes 1 - g in 64 bits, which is off by 2^-53 e^g of itself)
    gate = torch.linspace(-60.0, 20.0, count)[torch.randperm(count, generator=torch.Generator().manual_seed(7))]
    gate = (gate if kind == "row" else gate.view(n, d)).to(DT[dtype]).cuda()
    for post in (True, False):
        kw = dict(w_post=w1, post=post, gate=gate, gate_fn="sigmoid", alpha=0.75, eps=EPS)
        Y, H = sn.sn_block_norm(X, R, w, **kw)
        _check_forward(Y, H, X, R, w, w1, post, gate, "sigmoid", 0.75, dtype, f"post={post}")
        gw, gw1, dg = (torch.zeros(d, device="cuda") for _ in range(3))
        r = sn.sn_block_norm_backward(X, H, dY, w, dH=dH, gw=gw, gw_post=gw1 if post else None,
                                      dgate=dg if kind == "row" else None, **kw)
        _check_backward((*r, gw, gw1 if post else None), 0.0 * host(gw), X, H, dY, w, w1, post, gate, "sigmoid", 0.75,
                        dH, dtype, f"post={post}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_past_every_exponential(dtype):
    """Infinite gates are 0 and 1 with no slope; a NaN gate stays in its own element of dX and dgate."""
    log(f"[block norm, infinite gates] {dtype}")
    n, d = 2, 64
    X, H, dH = (_mat(k, n, d, dtype) for k in (1, 2, 3))
    gate = torch.full((n, d), float("inf"), dtype=DT[dtype], device="cuda")
    gate[0, ::2], gate[1, 7] = -float("inf"), float("nan")
    dX, _, dg = sn.sn_block_norm_backward(X, H, None, post=False, gate=gate, gate_fn="sigmoid", dH=dH)
    ok = ~gate.isnan()
    assert torch.equal(dX[ok], torch.where(gate == float("inf"), dH, torch.zeros_like(dH))[ok])
    assert float(dg[ok].abs().max()) == 0.0 and bool(dX[1, 7].isnan()) and bool(dg[1, 7].isnan())
