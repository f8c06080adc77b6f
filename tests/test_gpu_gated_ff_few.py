"""Up to 384 float32 tokens of the gated feed-forward block and its dX, whose weights are multiplied as
they are, against the float64 oracle: both sides of every limit between the kernel's forms, lengths
shorter than a round of 64 and with every rest, columns at the edges of strips, slices.

Tolerance (u = 2^-24, K terms of sizes S): a sum is four chains of K / 4 terms at most, which are added,
and the slices after them, 16 (dX: 32) at most: u (K / 4 + 4 + 32) S.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import gated_ff as orc
from test_gpu_gated_ff import U, _mat, _near

pytestmark = pytest.mark.gpu

TOKENS = [1, 15, 16, 17, 32, 33, 48, 49, 80, 81, 96, 112, 113, 128, 129, 161, 256, 257, 273, 384]
LENGTHS = [(1, 4), (3, 5), (4, 63), (61, 64), (63, 65), (64, 66), (65, 127), (66, 128), (67, 129), (127, 130),
           (128, 257), (190, 1030), (512, 100), (1000, 12), (2049, 61), (4100, 36)]


def _tol(k, size):
    return U * (k / 4 + 36) * size


def _check(n, d, ff, pad, shift, act="silu"):
    X = _mat(n, n, d, "f32", pad, 1.0, shift)
    Wg, Wu = (_mat(s, d, ff, "f32", 2 * pad, d ** -0.5, shift) for s in (1, 2))
    out = torch.full((3, n, ff + 5), 7.0, device="cuda")
    H, G, Ut = sn.sn_gated_ff(X, Wg, Wu, act=act, out=out[0, :, :ff], out_g=out[1, :, :ff], out_u=out[2, :, :ff])
    x, wg, wu = host(X), host(Wg), host(Wu)
    h, g, u = orc.gated_ff(x, wg, wu, act)
    tg, tu = _tol(d, np.abs(x) @ np.abs(wg)), _tol(d, np.abs(x) @ np.abs(wu))
    _near(host(G), g, tg, "G")
    _near(host(Ut), u, tu, "U")
    th = 1.2 * tg * (np.abs(u) + tu) + np.abs(orc.act(act, g)[0]) * tu + np.abs(h) * U * (16 + 2 * g * g)
    _near(host(H), h, th, "H")
    assert bool((out[:, :, ff:] == 7.0).all())
    assert torch.equal(sn.sn_gated_ff(X, Wg, Wu, act=act), H)
    dH = _mat(5, n, ff, "f32", pad, 0.1, shift)
    dG, dU = (torch.empty(n, ff + pad, device="cuda")[:, :ff] for _ in range(2))
    room = torch.full((n, d + 3), 7.0, device="cuda")
    dX, _, _ = sn.sn_gated_ff_backward(X, Wg, Wu, G, Ut, dH, act=act, dG=dG, dU=dU, out=room[:, :d], want_gw=False)
    dg, du = host(dG), host(dU)
    ref, _, _ = orc.products_backward(x, wg, wu, dg, du)
    _near(host(dX), ref, _tol(ff, np.abs(dg) @ np.abs(wg).T + np.abs(du) @ np.abs(wu).T), "dX")
    assert bool((room[:, d:] == 7.0).all())
    again, _, _ = sn.sn_gated_ff_backward(X, Wg, Wu, G, Ut, dH, act=act, dG=dG, dU=dU)
    assert torch.equal(again, dX)


@pytest.mark.parametrize("n", TOKENS)
def test_tokens(n):
    log(f"[gated ff, f32] {n} tokens")
    _check(n, 200, 260, 0, 0)
    _check(n, 131, 197, 1, 3, "gelu")


@pytest.mark.parametrize("n", [5, 100, 200])
@pytest.mark.parametrize("d,ff", LENGTHS, ids=str)
def test_lengths(n, d, ff):
    log(f"[gated ff, f32] {n} x {d} x {ff}")
    _check(n, d, ff, 0, 0)
    _check(n, d, ff, 3, 1, "relu")


@pytest.mark.parametrize("n,d,ff", [(130, 520, 8200), (384, 2050, 4100), (20, 4097, 8195)], ids=str)
def test_large(n, d, ff):
    """More workgroups than CUs, and slices of both products."""
    log(f"[gated ff, f32] {n} x {d} x {ff}")
    _check(n, d, ff, 1, 1)


@pytest.mark.parametrize("which", ["X", "weights"])
def test_offsets_past_32_bits(which):
    """Rows so far apart that their elements' numbers pass 2^31."""
    log(f"[gated ff, f32] far rows of {which}")
    n, d, ff = 300, 2100, 96
    far = 1 << 23 if which == "X" else 0
    room = torch.empty(n * (far or d), device="cuda")
    X = room.view(n, far or d)[:, :d]
    X.copy_(_mat(1, n, d, "f32"))
    ld = (1 << 20) + 40 if which == "weights" else 2 * ff
    W = torch.empty(d * ld, device="cuda").view(d, ld)[:, :2 * ff]
    W.copy_(_mat(2, d, 2 * ff, "f32", 0, d ** -0.5))
    H, G, Ut = sn.sn_gated_ff(X, W[:, :ff], W[:, ff:], save=True)
    near = sn.sn_gated_ff(X.clone(), W[:, :ff].clone(), W[:, ff:].clone(), save=True)
    assert all(torch.equal(a, b) for a, b in zip((H, G, Ut), near))
    dH = _mat(3, n, ff, "f32", 0, 0.1)
    a = sn.sn_gated_ff_backward(X, W[:, :ff], W[:, ff:], G, Ut, dH)
    b = sn.sn_gated_ff_backward(X.clone(), W[:, :ff].clone(), W[:, ff:].clone(), G, Ut, dH)
    assert all(torch.equal(s, t) for s, t in zip(a, b))


@pytest.mark.parametrize("n,d,ff", [(20, 2000, 70), (130, 1300, 200), (384, 640, 1000)], ids=str)
def test_calls_keep_to_their_workspace(n, d, ff):
    """Slices' parts lie in the workspace; behind it nothing is written."""
    log(f"[gated ff, f32, workspace] {n} x {d} x {ff}")
    X, Wg, Wu = _mat(1, n, d, "f32"), _mat(2, d, ff, "f32", 0, d ** -0.5), _mat(3, d, ff, "f32", 0, d ** -0.5)
    f = sn.sn_gated_ff_workspace_bytes(n, d, ff, d, ff, 0, True)
    b = sn.sn_gated_ff_backward_workspace_bytes(n, d, ff, d, ff, ff, 0, True)
    assert f > 0 and b > 0
    H, G, Ut = sn.sn_gated_ff(X, Wg, Wu, save=True)
    for need, call, want in ((f, lambda ws: sn.sn_gated_ff(X, Wg, Wu, save=True, workspace=ws), (H, G, Ut)),
                             (b, lambda ws: sn.sn_gated_ff_backward(X, Wg, Wu, G, Ut, H, workspace=ws),
                              sn.sn_gated_ff_backward(X, Wg, Wu, G, Ut, H))):
        room = torch.full((need + (1 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
        got = call(room[:need])
        assert bool((room[need:] == 0x5A).all()) and all(torch.equal(s, t) for s, t in zip(got, want))


def test_two_streams_at_once():
    log("[gated ff, f32, streams]")
    n, d, ff = 200, 512, 1100
    Wg, Wu = _mat(2, d, ff, "f32", 0, d ** -0.5), _mat(3, d, ff, "f32", 0, d ** -0.5)
    X = [_mat(k, n, d, "f32") for k in (4, 5)]

    def calls(x, stream=None):
        H, G, Ut = sn.sn_gated_ff(x, Wg, Wu, save=True, stream=stream)
        return (H, G, Ut, *sn.sn_gated_ff_backward(x, Wg, Wu, G, Ut, H, stream=stream))
    want = [calls(x) for x in X]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [calls(x, s) for x, s in zip(X, streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(s, t) for s, t in zip(a, b))
