"""GPU parity of the root-mean-square norm, its 8-bit form and its backward
through the binding against the float64 oracle.

Tolerances (u = 2^-24).  A row's sum of d squares is float32: at most d / 64 + 32
terms per thread, then a tree of at most 16 levels; half of its relative error
reaches the norm's factor, so with s = d / 64 + 48:
  * y:   |y| u (s / 2 + 8)
  * scales: the same of the largest |y|;  codes: that of a value within
    |y / s| u (s + 20), twice, of y / s
  * dX:  u [ (rho |u|)(s / 2 + 12) + |h| rho^3 mean|u h| (5 s / 2 + 20) + 2 |dh| ]
  * gw:  u [ s / 2 + 12 + rows / 256 + 64 ] sum over rows |dy h rho|
and for bf16 outputs their own rounding, 2^-8 of the value.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import rmsnorm as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
# one element, ragged pieces, both sides of each limit between the row layouts
# (64, 128, 256, 512, 1024, 2048, 4096 pieces of 4 floats or 8 bf16)
WIDTHS = [1, 3, 8, 127, 128, 129, 250, 512, 513, 1024, 1030, 1600, 2048, 2049, 4096, 4097, 8192,
          8200, 16384, 16400, 32768, 32777, 40000]


def _mat(seed, n, d, dtype, pad=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, d + pad, generator=g) * std).to(DT[dtype]).cuda()[:, :d]


def _gain(seed, d, dtype):
    g = torch.Generator().manual_seed(seed)
    return (1 + 0.2 * torch.randn(d, generator=g)).to(DT[dtype]).cuda()


def _h(t):
    return None if t is None else host(t)


def _near(got, ref, tol, what):
    err = np.abs(np.asarray(got, np.float64) - ref)
    tol = np.broadcast_to(tol, ref.shape) + 1e-37
    assert err.shape == ref.shape and np.isfinite(err).all(), what
    k = np.unravel_index(int(np.argmax(err - tol)), err.shape)
    assert (err <= tol).all(), f"{what} {k}: {got[k]!r}, {ref[k]!r}: {err[k]:.3g} over {tol[k]:.3g}"
    log(f"  {what}: ok, at most {float(np.max(err / tol)):.2g} of the bound")


def _own(ref, dtype):
    return 2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0


def _s(d):
    return d / 64 + 48


def _check_y(Y, H, X, w, R, dtype, what):
    y, h = orc.rmsnorm(_h(X), _h(w), _h(R), EPS)
    _near(host(Y), y, U * np.abs(y) * (_s(X.shape[1]) / 2 + 8) + _own(y, dtype), f"{what} Y")
    if R is not None:
        _near(host(H), h, U * np.abs(h) + _own(h, dtype), f"{what} H")


def _check_q(Q, S, X, w, R, group, what):
    y, _ = orc.rmsnorm(_h(X), _h(w), _h(R), EPS)
    d = y.shape[1]
    want = orc.scales(y, group)
    rel = U * (_s(d) / 2 + 12)
    _near(host(S), want, rel * want, f"{what} S")
    # the code of some value within the error of y / s: the exact one's where no
    # boundary is that near (a maximum 7 / 8 of a power of two puts bf16 rows on them)
    v, e = y / orc.spread(host(S), d, group), 2 * U * (_s(d) + 20)
    q = host(Q)
    assert np.isfinite(q).all()
    lo, hi = (orc.round_e4m3(np.clip(v * k, -448, 448)) for k in (1 - e, 1 + e))
    assert ((q == lo) | (q == hi)).all(), what
    log(f"  {what}: ok, {int((lo != hi).sum())} of {q.size} codes on a boundary")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward_matches_oracle(dtype, d):
    log(f"[rmsnorm] {dtype} d={d}")
    for n, pad, gain, res in ((1, 0, True, True), (5, 3, True, True), (6, 1, False, True),
                              (3, 8, True, False)):
        X, R = _mat(d, n, d, dtype, pad), _mat(d + 1, n, d, dtype, 2 * pad, 2.0) if res else None
        w = _gain(d, d, dtype) if gain else None
        what = f"n={n} pad={pad} gain={gain} res={res}"
        Y, H = sn.sn_rmsnorm(X, w, residual=R, eps=EPS)
        assert res or H is X
        _check_y(Y, H, X, w, R, dtype, what)
        for group in (0, 128):
            Q, S, H2 = sn.sn_rmsnorm_quant(X, w, residual=R, eps=EPS, group=group)
            assert torch.equal(H2, H)
            _check_q(Q, S, X, w, R, group, f"{what} group={group}")
        if res:  # in place of either operand, outputs with gaps
            for k in range(2):
                A, B = X.clone(), R.clone()
                out = torch.zeros(n, d + 5, dtype=X.dtype, device="cuda")
                Y2, H2 = sn.sn_rmsnorm(A, w, residual=B, eps=EPS, out=out[:, :d],
                                       resid_out=(A, B)[k])
                assert H2 is (A, B)[k] and torch.equal(H2, H) and torch.equal(Y2, Y)
                assert float(out[:, d:].abs().max()) == 0.0
            q = torch.zeros(n, d + 5, dtype=torch.uint8, device="cuda")
            s = torch.full((n, S.shape[1] + 2), 7.0, device="cuda")
            Q2, S2, _ = sn.sn_rmsnorm_quant(X, w, residual=R, eps=EPS, group=128,
                                            out=q.view(torch.float8_e4m3fn)[:, :d],
                                            scales=s[:, :S.shape[1]])
            assert torch.equal(Q2.contiguous().view(torch.uint8), Q.view(torch.uint8))
            assert torch.equal(S2, S) and int(q[:, d:].max()) == 0 and float(s[:, -2:].min()) == 7.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward_matches_oracle(dtype, d):
    log(f"[rmsnorm backward] {dtype} d={d}")
    for n, pad, gain, res in ((1, 0, True, True), (7, 3, True, True), (6, 1, False, False),
                              (3, 8, True, False)):
        H, dY = _mat(d, n, d, dtype, pad, 2.0), _mat(d + 1, n, d, dtype, 2 * pad, 0.1)
        dH = _mat(d + 2, n, d, dtype, pad, 0.1) if res else None
        w = _gain(d, d, dtype) if gain else None
        start = torch.linspace(-1, 1, d, device="cuda")
        gw = start.clone() if gain else None
        dX = sn.sn_rmsnorm_backward(H, dY, w, dH=dH, eps=EPS, gw=gw)
        _check_backward(dX, gw, start, H, dY, w, dH, dtype, f"n={n} pad={pad} gain={gain} res={res}")
        for on in (dY, dH):  # in place of either gradient
            if on is None:
                continue
            A, B = dY.clone(), None if dH is None else dH.clone()
            to = A if on is dY else B
            got = sn.sn_rmsnorm_backward(H, A, w, dH=B, eps=EPS, out=to)
            assert got is to and torch.equal(to, dX)


def _check_backward(dX, gw, start, H, dY, w, dH, dtype, what):
    h, dy, wv = host(H), host(dY), _h(w)
    n, d = h.shape
    ref, g = orc.rmsnorm_backward(h, dy, wv, _h(dH), EPS)
    rho = 1 / np.sqrt((h * h).mean(1, keepdims=True) + EPS)
    u = dy if wv is None else dy * wv
    s = _s(d)
    tol = rho * np.abs(u) * (s / 2 + 12) + \
        np.abs(h) * rho ** 3 * np.abs(u * h).mean(1, keepdims=True) * (5 * s / 2 + 20)
    if dH is not None:
        tol = tol + 2 * np.abs(host(dH))
    _near(host(dX), ref, U * tol + _own(ref, dtype), f"{what} dX")
    if gw is not None:
        tol = U * (s / 2 + 12 + n / 256 + 64) * np.abs(dy * h * rho).sum(0) + U * np.abs(host(start))
        _near(host(gw), host(start) + g, tol + U * np.abs(g), f"{what} gw")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("power,eps", [(-60, 0.0), (50, EPS)])
@pytest.mark.parametrize("d", [3, 130, 1600, 5000, 40000])
def test_backward_of_tiny_and_huge_rows(dtype, power, eps, d):
    """rho^3 = 2^180 or 2^-150 is no float32, the gradient is."""
    log(f"[rmsnorm backward of tiny and huge rows] {dtype} d={d} 2^{power}")
    H, dY, w = _mat(1, 5, d, dtype) * 2.0 ** power, _mat(2, 5, d, dtype), _gain(3, d, dtype)
    gw = torch.zeros(d, device="cuda")
    dX = sn.sn_rmsnorm_backward(H, dY, w, eps=eps, gw=gw)
    h, dy, u, s = host(H), host(dY), host(dY) * host(w), _s(d)
    ref, g = orc.rmsnorm_backward(h, dy, host(w), eps=eps)
    rho = 1 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    tol = rho * np.abs(u) * (s / 2 + 12) + \
        np.abs(h) * rho ** 3 * np.abs(u * h).mean(1, keepdims=True) * (5 * s / 2 + 20)
    _near(host(dX), ref, U * tol + _own(ref, dtype), "dX")
    _near(host(gw), g, U * ((s / 2 + 12 + 64) * np.abs(dy * h * rho).sum(0) + np.abs(g)), "gw")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(3001, 256), (2049, 1000), (1111, 4096)])
def test_many_rows(dtype, n, d):
    log(f"[rmsnorm many rows] {dtype} {n} x {d}")
    X, R, w = _mat(1, n, d, dtype), _mat(2, n, d, dtype), _gain(3, d, dtype)
    Y, H = sn.sn_rmsnorm(X, w, residual=R, eps=EPS)
    _check_y(Y, H, X, w, R, dtype, "forward")
    Q, S, _ = sn.sn_rmsnorm_quant(X, w, residual=R, eps=EPS, group=128)
    _check_q(Q, S, X, w, R, 128, "quant")
    gw = torch.zeros(d, device="cuda")
    dX = sn.sn_rmsnorm_backward(X, R, w, dH=Y, eps=EPS, gw=gw)
    _check_backward(dX, gw, torch.zeros(d), X, R, w, Y, dtype, "backward")
    again = torch.zeros(d, device="cuda")
    assert torch.equal(dX, sn.sn_rmsnorm_backward(X, R, w, dH=Y, eps=EPS, gw=again))
    assert torch.equal(gw, again)


@pytest.mark.parametrize("n,d", [(4096, 2055), (4097, 5003)])
def test_backward_of_many_odd_rows(n, d):
    """Rows of bf16 at odd elements, in an odd number of workgroups."""
    log(f"[rmsnorm backward of odd rows] {n} x {d}")
    H, dY, dH = (_mat(i, n, d, "bf16") for i in (1, 2, 3))
    w = _gain(4, d, "bf16")
    gw = torch.zeros(d, device="cuda")
    dX = sn.sn_rmsnorm_backward(H, dY, w, dH=dH, eps=EPS, gw=gw)
    _check_backward(dX, gw, torch.zeros(d), H, dY, w, dH, "bf16", "backward")


@pytest.mark.parametrize("d", [130, 1600, 5000, 40000])
def test_special_rows(d):
    """Zeros, tiny and huge rows, NaN and infinities: rows beside them are untouched."""
    log(f"[rmsnorm special rows] d={d}")
    for dtype in ("f32", "bf16"):
        X = _mat(4, 6, d, dtype).clone()
        X[0] = 0
        X[1] *= 2.0 ** -60
        X[2, d // 2] = float("nan")
        X[3, 1] = float("inf")
        X[4] *= 2.0 ** 50
        Y, _ = sn.sn_rmsnorm(X, eps=0.0 if d == 130 else EPS)
        y = host(Y)
        assert np.isnan(y[2]).all() and np.isnan(y[3, 1])
        if d != 130:
            assert (y[0] == 0).all()
        ref, _ = orc.rmsnorm(host(X)[[1, 4, 5]], eps=0.0 if d == 130 else EPS)
        got = y[[1, 4, 5]]
        if d == 130:  # 2^-60 squared is a float32; without eps the row is scaled up
            assert np.isnan(y[0]).all()
        _near(got, ref, U * np.abs(ref) * (_s(d) / 2 + 8) + _own(ref, dtype), dtype)
        for group in (0, 128):
            Q, S, _ = sn.sn_rmsnorm_quant(X, eps=EPS, group=group)
            q, s = host(Q), host(S)
            assert (q[0] == 0).all() and np.allclose(s[0], 2.0 ** -100 / 448, rtol=1e-6)
            assert np.isnan(q[2]).all() and np.isnan(s[2]).all()
            assert np.isnan(q[3, 1]) and np.isnan(s[3, 0])
            _check_q(Q[[5]], S[[5]], X[[5]], None, None, group, f"{dtype} group {group}")
    # a NaN gain spoils the columns of its own scale only
    w = torch.ones(d, device="cuda")
    w[0] = float("nan")
    Q, S, _ = sn.sn_rmsnorm_quant(_mat(5, 2, d, "f32"), w, group=128)
    assert np.isnan(host(Q)[:, :128]).all() and np.isnan(host(S)[:, 0]).all()
    assert np.isfinite(host(Q)[:, 128:]).all() and np.isfinite(host(S)[:, 1:]).all()


def test_offsets_past_two_to_the_31():
    log("[rmsnorm 2^31]")
    n, d = 300000, 8192
    X = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    X[-2:] = _mat(6, 2, d, "bf16")
    w = _gain(7, d, "bf16")
    Y, _ = sn.sn_rmsnorm(X, w)
    _check_y(Y[-2:], None, X[-2:], w, None, "bf16", "last rows")
    gw = torch.zeros(d, device="cuda")
    dX = sn.sn_rmsnorm_backward(X, X, w, gw=gw, out=Y)
    _check_backward(dX[-2:], None, None, X[-2:], X[-2:], w, None, "bf16", "last rows")


def test_gradient_against_differences():
    """<dX, v> + <gw, e> against central differences of <dY, y> along (v, e)."""
    log("[rmsnorm differences]")
    n, d, step = 5, 700, 2.0 ** -6
    X, R, w = _mat(1, n, d, "f32"), _mat(2, n, d, "f32"), _gain(3, d, "f32")
    dY, v, e = _mat(4, n, d, "f32"), _mat(5, n, d, "f32"), _gain(6, d, "f32")

    def f(k):
        return float((sn.sn_rmsnorm(X + k * v, w + k * e, residual=R)[0].double() * dY.double()).sum())

    _, H = sn.sn_rmsnorm(X, w, residual=R)
    gw = torch.zeros(d, device="cuda")
    dX = sn.sn_rmsnorm_backward(H, dY, w, gw=gw)
    have = float((dX.double() * v.double()).sum() + (gw.double() * e.double()).sum())
    want = (f(step) - f(-step)) / (2 * step)
    log(f"  {have:.5f} against {want:.5f}")
    scale = float(dY.double().norm() * v.double().norm()) / n ** 0.5
    assert abs(have - want) <= 1e-3 * scale


def test_refusals_streams_and_empty():
    log("[rmsnorm refusals]")
    X, R, w = _mat(1, 4, 96, "bf16"), _mat(2, 4, 96, "bf16"), _gain(3, 96, "bf16")
    gw = torch.zeros(96, device="cuda")
    wide = torch.zeros(4, 200, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(64, dtype=torch.uint8, device="cuda")
    for status, call in (
            (3, lambda: sn.sn_rmsnorm(X.half(), w)),
            (3, lambda: sn.sn_rmsnorm(X, w.float())),
            (2, lambda: sn.sn_rmsnorm(X, w[:95])),
            (2, lambda: sn.sn_rmsnorm(X, w, residual=R[:3])),
            (3, lambda: sn.sn_rmsnorm(X, w, residual=R.float())),
            (2, lambda: sn.sn_rmsnorm(X, w, eps=-1.0)),
            (2, lambda: sn.sn_rmsnorm(X, w, eps=float("nan"))),
            (2, lambda: sn.sn_rmsnorm(X.t(), w)),
            (2, lambda: sn.sn_rmsnorm(X.cpu(), w)),
            (5, lambda: sn.sn_rmsnorm(X, w, residual=R, out=R)),
            (5, lambda: sn.sn_rmsnorm(X, w, out=X)),
            (5, lambda: sn.sn_rmsnorm(wide[:, :96], w, residual=R, resid_out=wide[:, 50:146])),
            (8, lambda: sn.sn_rmsnorm_quant(X, w, group=64)),
            (3, lambda: sn.sn_rmsnorm_quant(X, w, out=torch.zeros(4, 96, dtype=torch.uint8, device="cuda"))),
            (2, lambda: sn.sn_rmsnorm_quant(X, w, group=128, scales=torch.zeros(4, 2, device="cuda"))),
            (3, lambda: sn.sn_rmsnorm_backward(X, R.float(), w)),
            (2, lambda: sn.sn_rmsnorm_backward(X, R, w, gw=gw[:5])),
            (2, lambda: sn.sn_rmsnorm_backward(X, R, w, gw=gw.bfloat16())),
            (5, lambda: sn.sn_rmsnorm_backward(X, R, w, out=X)),
            (9, lambda: sn.sn_rmsnorm_backward(X, R, w, gw=gw, workspace=ws))):
        with pytest.raises(sn.SnError) as e:
            call()
        assert e.value.status == status, e.value
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = sn.sn_rmsnorm(X, w, residual=R, stream=s)
    b = sn.sn_rmsnorm_quant(X, w, residual=R, stream=s)
    c = sn.sn_rmsnorm_backward(X, R, w, gw=gw, stream=s)
    s.synchronize()
    assert torch.equal(a[0], sn.sn_rmsnorm(X, w, residual=R)[0])
    assert torch.equal(b[1], sn.sn_rmsnorm_quant(X, w, residual=R)[1])
    g2 = torch.zeros(96, device="cuda")
    assert torch.equal(c, sn.sn_rmsnorm_backward(X, R, w, gw=g2)) and torch.equal(gw, g2)
    assert sn.sn_rmsnorm(X[:0], w)[0].shape == (0, 96)
    assert sn.sn_rmsnorm_backward(X[:0], R[:0], w, gw=gw).shape == (0, 96)
    assert torch.equal(gw, g2)


def test_in_a_graph():
    log("[rmsnorm graph]")
    X, R, w = _mat(1, 300, 1600, "bf16"), _mat(2, 300, 1600, "bf16"), _gain(3, 1600, "bf16")
    gw = torch.zeros(1600, device="cuda")
    keep = {}

    def step():
        gw.zero_()
        Y, H = sn.sn_rmsnorm(X, w, residual=R)
        Q, S, _ = sn.sn_rmsnorm_quant(X, w, residual=R, group=128)
        keep["t"] = (Y, H, Q.view(torch.uint8), S, sn.sn_rmsnorm_backward(H, Y, w, dH=R, gw=gw), gw)

    step()
    want = [t.clone() for t in keep["t"]]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in keep["t"]:
            t.fill_(3)
        sn.sn_rmsnorm(X[:3], w)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, keep["t"]):
            assert torch.equal(x, y)
