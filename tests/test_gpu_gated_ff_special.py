"""Large, small and special values in the gated feed-forward block's products, forward and backward,
on every path by the number of tokens.

Sums of one term that is not zero are that term: float32 as it is where the operands are multiplied as
they are, and bf16 everywhere.  Where float32 operands are multiplied in three bf16 parts, the matrix cores
take operands and sums below 2^-126 as 0: each part (stored as large as 2^14 times itself) loses less
than 2^-126 by that, and so does the sum at each of its two steps from one part to the next, 5 x 2^-126
in all, which a value of 2^-100 or more does not feel.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SCALES = (1.0, 1e30, 1e-30, 3.0e38, 1e-37)
AS_THEY_ARE = 384  # float32 tokens, forward and in dX; weights' gradients have no such path


def _tiny(dtype, n, scale, most):
    return 5 * 2.0 ** -126 if dtype == "f32" and n > most and scale < 2.0 ** -100 else 0.0


def _mat(seed, n, d, dtype):
    return torch.randn(n, d, generator=torch.Generator().manual_seed(seed)).to(DT[dtype]).cuda()


def _alike(got, ref):
    """The same bits, NaN as NaN."""
    return torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.nan_to_num(7.0), ref.nan_to_num(7.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 40, 128, 129, 300, 385, 700])
def test_forward(dtype, n):
    log(f"[gated ff, special] {dtype} {n} tokens")
    d, ff = 72, 136
    one = torch.zeros(d, ff, dtype=DT[dtype], device="cuda")
    one[0] = 1.0
    for scale in SCALES:
        Z = torch.zeros(n, d, dtype=DT[dtype], device="cuda")
        Z[:, 0] = torch.linspace(0.5, 1.0, n, device="cuda") * scale
        H, G, _ = sn.sn_gated_ff(Z, one, one * 0.0, act="relu", save=True)
        tiny = _tiny(dtype, n, scale, AS_THEY_ARE)
        assert np.abs(host(G) - host(Z[:, :1])).max() <= tiny and float(H.abs().max()) == 0.0, scale
    X, Wg, Wu = _mat(1, n, d, dtype), _mat(2, d, ff, dtype), _mat(3, d, ff, dtype)
    good = sn.sn_gated_ff(X, Wg, Wu, save=True)
    t, keep = n // 2, [i for i in range(n) if i != n // 2]
    for value in ("nan", "inf"):
        bad = X.clone()
        bad[t, 3] = float(value)
        got = sn.sn_gated_ff(bad, Wg, Wu, save=True)
        for a, b in zip(got, good):
            assert torch.equal(a[keep], b[keep]), value
        for a in got[1:]:
            assert not bool(a[t].isfinite().any()), value
    W = Wu.clone()
    W[5, 77] = float("nan")
    got = sn.sn_gated_ff(X, Wg, W, save=True)
    cols = [c for c in range(ff) if c != 77]
    assert bool(got[2][:, 77].isnan().all()) and bool(got[0][:, 77].isnan().all())
    assert torch.equal(got[2][:, cols], good[2][:, cols]) and torch.equal(got[1], good[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 64, 129, 300, 385, 700])
def test_backward_ranges(dtype, n):
    """relu, G = 1 and U = 0: dU is dH, dG is 0, and dX and gWu are one term each."""
    log(f"[gated ff backward, range] {dtype} {n} tokens")
    d, ff = 72, 136
    G, U = torch.ones(n, ff, dtype=DT[dtype], device="cuda"), torch.zeros(n, ff, dtype=DT[dtype], device="cuda")
    X, W = torch.zeros(n, d, dtype=DT[dtype], device="cuda"), torch.zeros(d, ff, dtype=DT[dtype], device="cuda")
    X[n // 3] = 1.0
    W[:, 0] = 1.0
    for scale in SCALES:
        dH = torch.zeros(n, ff, dtype=DT[dtype], device="cuda")
        dH[:, 0] = torch.linspace(0.5, 1.0, n, device="cuda") * scale
        dX, gWg, gWu = sn.sn_gated_ff_backward(X, W, W, G, U, dH, act="relu")
        assert np.abs(host(dX) - host(dH[:, :1])).max() <= _tiny(dtype, n, scale, AS_THEY_ARE), scale
        tiny = _tiny(dtype, n, scale, 0)
        assert np.abs(host(gWu)[:, 0] - float(dH[n // 3, 0])).max() <= tiny, scale
        assert float(gWg.abs().max()) == 0.0 and float(gWu[:, 1:].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 64, 129, 300, 385, 700])
def test_backward_special_values(dtype, n):
    """A NaN or an infinity enters the results that are made with it, and no others change."""
    log(f"[gated ff backward, special] {dtype} {n} tokens")
    d, ff, t, j, c = 72, 136, n // 2, 7, 100
    X, Wg, Wu = _mat(1, n, d, dtype), _mat(2, d, ff, dtype), _mat(3, d, ff, dtype)
    G, U, dH = _mat(4, n, ff, dtype), _mat(5, n, ff, dtype), _mat(6, n, ff, dtype)
    G[t, c] = 1.5  # no zero of the derivative
    good = sn.sn_gated_ff_backward(X, Wg, Wu, G, U, dH)
    rows, dims, cols = ([i for i in range(k) if i != at] for k, at in ((n, t), (d, j), (ff, c)))
    for value in (float("nan"), float("inf")):
        bad = dH.clone()
        bad[t, c] = value
        dX, gWg, gWu = sn.sn_gated_ff_backward(X, Wg, Wu, G, U, bad)
        assert not bool(dX[t].isfinite().any()) and torch.equal(dX[rows], good[0][rows])
        for a, b in ((gWg, good[1]), (gWu, good[2])):
            assert not bool(a[:, c].isfinite().any()) and torch.equal(a[:, cols], b[:, cols])
        bad = X.clone()
        bad[t, j] = value
        dX, gWg, gWu = sn.sn_gated_ff_backward(bad, Wg, Wu, G, U, dH)
        assert torch.equal(dX, good[0])
        for a, b in ((gWg, good[1]), (gWu, good[2])):
            assert not bool(a[j].isfinite().any()) and torch.equal(a[dims], b[dims])
        bad = Wg.clone()
        bad[j, c] = value
        dX, gWg, gWu = sn.sn_gated_ff_backward(X, bad, Wu, G, U, dH)
        assert not bool(dX[:, j].isfinite().any()) and torch.equal(dX[:, dims], good[0][:, dims])
        assert _alike(gWg, good[1]) and _alike(gWu, good[2])
