"""The norm at its limits: 8-bit codes on the boundaries between two codes, against
the quotient that the header names, code for code."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import rmsnorm as orc

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _codes(v):
    return orc.round_e4m3(np.clip(v.astype(np.float64), -448, 448))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [6, 40, 130, 512, 1600, 5000, 16400])
def test_codes_are_those_of_the_quotient(dtype, d):
    """Whole numbers up to 28 = 7/8 of 32, so that odd ones above 16 lie on a boundary
    (448 * 17 / 28 = 272, between 256 and 288), to the last bits of y and s.  Their
    squares' sum is exact in any order (at most 28^2 * 16400 < 2^24), so that y is the
    same float32 in every form of the call, and sn_rmsnorm in float32 returns it."""
    log(f"[rmsnorm codes] {dtype} d={d}")
    g = torch.Generator().manual_seed(d)
    n = 96
    X = torch.randint(-28, 29, (n, d), generator=g).float()
    X[:, ::5] = 28.0  # each scale's columns reach it
    X[:, 1::7] = torch.randint(8, 14, (n, len(range(1, d, 7))), generator=g).float() * 2 + 1
    X[:, 3] = -0.0
    X = X.cuda()
    differs = 0
    for w in (None, (1 + 0.2 * torch.randn(d, generator=g)).bfloat16().cuda()):
        Y, _ = sn.sn_rmsnorm(X, None if w is None else w.float(), eps=0.0)
        y = Y.cpu().numpy()
        for group in (0, 128):
            Q, S, _ = sn.sn_rmsnorm_quant(X.to(DT[dtype]), None if w is None else w.to(DT[dtype]),
                                          eps=0.0, group=group)
            cuts = list(range(0, d, group or d)) + [d]
            s = np.stack([np.abs(y[:, i:j]).max(1) for i, j in zip(cuts, cuts[1:])], 1) / np.float32(448)
            assert s.dtype == np.float32 and np.array_equal(S.cpu().numpy(), s)
            each = orc.spread(s, d, group)
            want, q = _codes(y / each), host(Q)
            assert np.array_equal(q, want), f"{int((q != want).sum())} of {q.size} codes"
            assert np.array_equal(np.signbit(q), np.signbit(want))
            if w is None:
                differs += int((_codes(y * (np.float32(1) / each)) != want).sum())
    # a product with the rounded reciprocal would not do
    log(f"  ok; a product with 1 / s has {differs} other codes")
    assert differs > 0 or d < 1000


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_codes_beside_infinities(dtype):
    """A gain that takes one value past float32's range makes its scale infinite: that
    value's quotient is NaN, every other one's 0, and other scales are untouched."""
    log(f"[rmsnorm codes beside infinities] {dtype}")
    for d in (300, 40000):
        X = torch.ones(3, d, dtype=DT[dtype], device="cuda")
        X[1, 5] = -2.0 ** 20  # about sqrt(d) after the norm
        w = torch.ones(d, dtype=DT[dtype], device="cuda")
        w[5] = torch.finfo(DT[dtype]).max
        Q, S, _ = sn.sn_rmsnorm_quant(X, w, group=128)
        q, s = host(Q), host(S)
        assert np.isinf(s[1, 0]) and np.isfinite(s[[0, 2]]).all() and np.isfinite(s[1, 1:]).all()
        assert np.isnan(q[1, 5]) and (np.delete(q[1, :128], 5) == 0).all()
        assert np.isfinite(q[[0, 2]]).all() and np.isfinite(q[1, 128:]).all()
        q = host(sn.sn_rmsnorm_quant(X, w)[0])
        assert np.isnan(q[1, 5]) and (np.delete(q[1], 5) == 0).all() and np.isfinite(q[[0, 2]]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gain_gradient_past_2_32_threads(dtype):
    """2^27 + 77 columns: the gain gradient's workgroups of 1024 threads for 32 columns
    take more than one grid dimension has.  Rows of ones with eps = 0, whose squares' sum
    is exact, so that rho is 1 to its last bits and gw the rows' sum of dy."""
    log(f"[rmsnorm gain gradient, 2^27 columns] {dtype}")
    n, d = 2, (1 << 27) + 77
    H = torch.ones(n, d, dtype=DT[dtype], device="cuda")
    dY = torch.zeros_like(H)
    gw = torch.ones(d, device="cuda")
    at = torch.tensor([0, 31, 1 << 20, (1 << 25) + 1, (1 << 27) - 1, 1 << 27, d - 1], device="cuda")
    dY[0, at], dY[1, at] = 2.0, -4.0
    dY[:, 5] = 6.0
    sn.sn_rmsnorm_backward(H, dY, eps=0.0, gw=gw)
    want = torch.ones(d, device="cuda")
    want[at], want[5] = -1.0, 13.0
    assert float((gw - want).abs().max()) <= 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [5, 300, 4096, 8190, 40000])
def test_largest_and_smallest_rows(dtype, d):
    """Rows of +-2^p on both sides of a sum of squares of 2^128, and the smallest ones.
    Inside, y is the sign to the rounding of rho (float32 sums of equal powers of two,
    at most d / 64 + 48 roundings, half of their error) and of a bf16 output."""
    log(f"[rmsnorm largest and smallest rows] {dtype} d={d}")
    u = 2.0 ** -24
    p = max(q for q in range(70) if d * 4.0 ** q < 2.0 ** 128)
    g = torch.Generator().manual_seed(d)
    sign = torch.randint(0, 2, (2, d), generator=g).float() * 2 - 1
    tol = u * (d / 128 + 40) + (2.0 ** -8 if dtype == "bf16" else 0.0)
    H = torch.stack([sign[0] * 2.0 ** p, sign[1] * 2.0 ** (p + 1)]).to(DT[dtype]).cuda()
    for w in (None, torch.full((d,), 0.5, dtype=DT[dtype], device="cuda")):
        k = 1.0 if w is None else 0.5
        Y, _ = sn.sn_rmsnorm(H, w)
        assert np.abs(host(Y)[0] - k * sign[0].numpy()).max() <= tol * k and float(Y[1].abs().max()) == 0.0
        Q, S, _ = sn.sn_rmsnorm_quant(H, w)
        assert np.abs(host(Q)[0] * host(S)[0] - k * sign[0].numpy()).max() <= k * u * (d / 128 + 48)
        assert float(Q[1].float().abs().max()) == 0.0
    # dx = rho (u - n mean(u n)), |n| = 1: at most the roundings of rho, of the mean (float32
    # over d terms) and of five operations, of |u| + mean |u| < 2
    dY = torch.rand(2, d, generator=g).to(DT[dtype]).cuda()
    dH = torch.randn(2, d, generator=g).to(DT[dtype]).cuda()
    gw = torch.ones(d, device="cuda")
    dX = sn.sn_rmsnorm_backward(H, dY, gw=gw)
    ref, gref = orc.rmsnorm_backward(host(H), host(dY))
    err = np.abs(host(dX)[0] - ref[0]) / 2.0 ** -p
    own = 2.0 ** -8 * np.abs(ref[0]) * 2.0 ** p if dtype == "bf16" else 0.0
    assert (err <= 2 * u * (d / 64 + 60) + own).all()
    assert float(dX[1].abs().max()) == 0.0
    # only the first row counts: |dy n| < 1
    want = 1.0 + host(dY)[0] * sign[0].numpy()
    assert np.abs(host(gw) - want).max() <= u * (d / 128 + 48)
    assert torch.equal(sn.sn_rmsnorm_backward(H, dY, dH=dH)[1], dH[1])
    # the small end: 2^-62 has its bits without eps, 2^-80 with one
    for power, eps in ((-62, 0.0), (-80, 1e-6), (-80, 2.0 ** -100)):
        X = (sign * 2.0 ** power).to(DT[dtype]).cuda()
        ref = sign.numpy() * 2.0 ** power / np.sqrt(4.0 ** power + float(np.float32(eps)))
        Y, _ = sn.sn_rmsnorm(X, eps=eps)
        assert (np.abs(host(Y) - ref) <= tol * np.abs(ref)).all(), power
    Y, _ = sn.sn_rmsnorm(X, eps=0.0)
    assert np.isinf(host(Y)).all() and bool(torch.isnan(sn.sn_rmsnorm(0 * X, eps=0.0)[0]).all())
