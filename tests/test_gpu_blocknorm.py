"""GPU parity of the block norm and its backward against the float64 oracle.

Tolerances (u = 2^-24).  A row's sum of d terms is float32: at most d / 64 + 32 terms per thread,
then a tree of at most 16 levels; with s = d / 64 + 48:
  * a norm's factor: u (s / 2 + 4) of itself; a sigmoid: 8 u of itself (expf, an addition, a
    division), its derivative 16 u
  * h:   |g z| u (s / 2 + 16) + 2 u |alpha r| + u |h|
  * y:   |y| u (s / 2 + 8), and through h: |w| rho tol(h) + |y| mean(|h| tol(h)) rho^2
  * dh:  u [ (rho |u|)(s / 2 + 12) + |h| rho^3 mean|u h| (5 s / 2 + 20) + 2 |dH| + 2 |dh| ]
  * dg, dz and what follows: tol(dh) times the factors, and u (s / 2 + 24) of the value
  * dX:  q (tol(v) + |m| mean(tol(v) |m|)) + u [ q |v| (s / 2 + 12) + q |m| mean|v m| (5 s / 2 + 20) ]
  * sums over rows: the rows' tolerances, and u (rows / 256 + 64) of the sum of sizes
and for bf16 outputs their own rounding, 2^-8 of the value.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import blocknorm as orc

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
# one element, ragged pieces, both sides of each limit between the row layouts
WIDTHS = [1, 3, 8, 127, 250, 256, 513, 1024, 1030, 1600, 2048, 2049, 4097, 8192, 8200, 16400, 32777]
GATES = [(None, "none"), ("row", "none"), ("row", "sigmoid"), ("token", "none"), ("token", "sigmoid")]


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


def _check_forward(Y, H, X, R, w, w1, post, gate, fn, alpha, dtype, what):
    y, h = orc.block_norm(_h(X), _h(R), _h(w), _h(w1), post, _h(gate), fn, alpha, EPS)
    s, gz = _s(X.shape[1]), h - alpha * _h(R)
    th = np.abs(gz) * U * (s / 2 + 16) + 2 * U * np.abs(alpha * _h(R)) + U * np.abs(h)
    _near(host(H), h, th + _own(h, dtype), f"{what} H")
    if Y is None:
        return
    rho = 1 / np.sqrt((h * h).mean(1, keepdims=True) + EPS)
    gain = 1.0 if w is None else np.abs(_h(w))
    ty = gain * rho * th + np.abs(y) * (np.abs(h) * th).mean(1, keepdims=True) * rho ** 2
    _near(host(Y), y, ty + np.abs(y) * U * (s / 2 + 8) + _own(y, dtype), f"{what} Y")


def _check_backward(got, starts, X, H, dY, w, w1, post, gate, fn, alpha, dH, dtype, what):
    dX, dR, dgate, gw, gw1 = got
    x, h = _h(X), _h(H)
    n, d = x.shape
    ref = orc.block_norm_backward(x, h, _h(dY), _h(w), _h(w1), post, _h(gate), fn, alpha, _h(dH), EPS)
    s, rows = _s(d), U * (n / 256 + 64)
    mean = lambda a: a.mean(1, keepdims=True)  # noqa: E731
    rho = 1 / np.sqrt(mean(h * h) + EPS)
    dy = np.zeros_like(x) if dY is None else _h(dY)
    u = np.abs(dy * (1.0 if w is None else _h(w)))
    tdh = U * (rho * u * (s / 2 + 12) + np.abs(h) * rho ** 3 * mean(u * np.abs(h)) * (2.5 * s + 20) +
               2 * np.abs(ref["dh"]))
    if dH is not None:
        tdh = tdh + 2 * U * np.abs(_h(dH))
    _near(host(dR), ref["dR"], abs(alpha) * tdh + U * np.abs(ref["dR"]) + _own(ref["dR"], dtype),
          f"{what} dR")
    g, slope = orc.gate_values(_h(gate), fn)
    q = 1 / np.sqrt(mean(x * x) + EPS) if post else 1.0
    m = x * q
    w1h = 1.0 if w1 is None or not post else _h(w1)
    if gate is not None:
        tdg = np.abs(m * w1h * slope) * tdh + np.abs(ref["dgate"]) * U * (s / 2 + 24)
        if gate.dim() == 2:
            _near(host(dgate), ref["dgate"], tdg + _own(ref["dgate"], dtype), f"{what} dgate")
        else:
            want = ref["dgate"].sum(0) + starts
            size = np.abs(ref["dgate"]).sum(0) + np.abs(starts)
            _near(host(dgate), want, tdg.sum(0) + rows * size + U * np.abs(want), f"{what} dgate")
    dz = ref["dh"] * g
    tdz = np.abs(g) * tdh + np.abs(dz) * 12 * U
    if not post:
        _near(host(dX), ref["dX"], tdz + _own(ref["dX"], dtype), f"{what} dX")
    else:
        v, tv = np.abs(dz * w1h), np.abs(w1h) * tdz + 2 * U * np.abs(dz * w1h)
        tol = q * (tv + np.abs(m) * mean(tv * np.abs(m))) + \
            U * (q * v * (s / 2 + 12) + q * np.abs(m) * mean(v * np.abs(m)) * (2.5 * s + 20))
        _near(host(dX), ref["dX"], tol + _own(ref["dX"], dtype), f"{what} dX")
        if gw1 is not None:
            each = np.abs(dz * m)
            tol = (np.abs(m) * tdz + each * U * (s / 2 + 12)).sum(0) + rows * (each.sum(0) + np.abs(starts))
            want = ref["gw_post"] + starts
            _near(host(gw1), want, tol + U * np.abs(want), f"{what} gw_post")
    if gw is not None:
        each = np.abs(dy * h * rho)
        want = ref["gw"] + starts
        _near(host(gw), want, (each * U * (s / 2 + 12)).sum(0) + rows * (each.sum(0) + np.abs(starts)) +
              U * np.abs(want), f"{what} gw")


def _gate_of(kind, n, d, dtype, pad):
    if kind is None:
        return None
    return _gain(d + 9, d, dtype) if kind == "row" else _mat(d + 9, n, d, dtype, pad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_forward_matches_oracle(dtype, d):
    log(f"[block norm] {dtype} d={d}")
    for k, (kind, fn) in enumerate(GATES):
        for post in (True, False):
            n, pad, gains = (1, 5, 6)[k % 3], (0, 3, 8)[(k + post) % 3], k != 3
            X, R = _mat(d, n, d, dtype, pad), _mat(d + 1, n, d, dtype, 2 * pad, 2.0)
            w, w1 = (_gain(d, d, dtype), _gain(d + 2, d, dtype)) if gains else (None, None)
            gate, alpha = _gate_of(kind, n, d, dtype, pad), (1.0, 0.75, -1.25)[k % 3]
            kw = dict(w_post=w1, post=post, gate=gate, gate_fn=fn, alpha=alpha, eps=EPS)
            Y, H = sn.sn_block_norm(X, R, w, **kw)
            what = f"n={n} pad={pad} gate={kind} {fn} post={post}"
            _check_forward(Y, H, X, R, w, w1, post, gate, fn, alpha, dtype, what)
            none, H2 = sn.sn_block_norm(X, R, w, next_norm=False, **kw)
            assert none is None and torch.equal(H2, H)
            for i in range(2):  # in place of either operand, outputs with gaps
                A, B = X.clone(), R.clone()
                out = torch.zeros(n, d + 5, dtype=X.dtype, device="cuda")
                Y2, H2 = sn.sn_block_norm(A, B, w, out=out[:, :d], resid_out=(A, B)[i], **kw)
                assert H2 is (A, B)[i] and torch.equal(H2, H) and torch.equal(Y2, Y)
                assert torch.equal((B, A)[i], (R, X)[i]) and float(out[:, d:].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_backward_matches_oracle(dtype, d):
    log(f"[block norm backward] {dtype} d={d}")
    for k, (kind, fn) in enumerate(GATES):
        for post in (True, False):
            n, pad, gains = (1, 7, 6)[k % 3], (0, 3, 8)[(k + post) % 3], k != 3
            X, H = _mat(d, n, d, dtype, pad), _mat(d + 1, n, d, dtype, pad, 2.0)
            dY = None if k == 4 and post else _mat(d + 2, n, d, dtype, 2 * pad, 0.1)
            dH = None if k == 1 else _mat(d + 3, n, d, dtype, pad, 0.1)
            w, w1 = (_gain(d, d, dtype), _gain(d + 4, d, dtype)) if gains else (None, None)
            gate, alpha = _gate_of(kind, n, d, dtype, pad), (1.0, 0.75, -1.25)[k % 3]
            start = torch.linspace(-1, 1, d, device="cuda")
            kw = dict(w_post=w1, post=post, gate=gate, gate_fn=fn, alpha=alpha, dH=dH, eps=EPS)

            def run(**more):
                gw = start.clone() if dY is not None else None
                gw1 = start.clone() if post else None
                more.setdefault("dgate", start.clone() if kind == "row" else None)
                r = sn.sn_block_norm_backward(X, H, dY, w, gw=gw, gw_post=gw1, **{**kw, **more})
                return (*r, gw, gw1)
            got = run()
            what = f"n={n} pad={pad} gate={kind} {fn} post={post} dY={dY is not None}"
            _check_backward(got, host(start), X, H, dY, w, w1, post, gate, fn, alpha, dH, dtype, what)
            # in place of the gradients, and of the gate
            more = {}
            if dH is not None and dY is not None:
                a, b = dY.clone(), dH.clone()
                r = sn.sn_block_norm_backward(X, H, a, w, out=a, resid_out=b, **{**kw, "dH": b})
                assert r[0] is a and r[1] is b and torch.equal(a, got[0]) and torch.equal(b, got[1])
                assert kind == "token" or r[2] is None
            x = X.clone()
            more = {"gate": gate.clone()} if kind == "token" else {}
            r = sn.sn_block_norm_backward(x, H, dY, w, out=x, dgate=more.get("gate"), **{**kw, **more})
            assert r[0] is x and torch.equal(x, got[0]) and torch.equal(r[1], got[1])
            assert kind != "token" or torch.equal(r[2], got[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(1300, 200), (2500, 2048), (1100, 4100), (600, 20000)])
def test_many_rows(dtype, n, d):
    """Every workgroup takes several rows; the sums are the same every time."""
    log(f"[block norm, many rows] {dtype} {n} x {d}")
    X, H = _mat(1, n, d, dtype), _mat(2, n, d, dtype, 0, 2.0)
    dY, dH = _mat(3, n, d, dtype, 0, 0.1), _mat(4, n, d, dtype, 0, 0.1)
    w, w1, gate = (_gain(k, d, dtype) for k in range(3))
    Y, R = sn.sn_block_norm(X, H, w, w_post=w1, gate=gate, gate_fn="sigmoid", alpha=0.5)
    _check_forward(Y, R, X, H, w, w1, True, gate, "sigmoid", 0.5, dtype, "forward")

    def run():
        gw, gw1, dg = (torch.zeros(d, device="cuda") for _ in range(3))
        r = sn.sn_block_norm_backward(X, H, dY, w, w_post=w1, gate=gate, gate_fn="sigmoid", alpha=0.5,
                                      dH=dH, gw=gw, gw_post=gw1, dgate=dg)
        return (*r, gw, gw1)
    got = run()
    _check_backward(got, np.zeros(d), X, H, dY, w, w1, True, gate, "sigmoid", 0.5, dH, dtype, "backward")
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(got, run()))


def test_extreme_gates_and_rows():
    """Sigmoids of infinities are 0 and 1; a row of zeros has z = 0; NaN stays in its row."""
    log("[block norm, extremes]")
    d = 64
    X, R = torch.ones(4, d, device="cuda"), torch.ones(4, d, device="cuda")
    gate = torch.full((d,), float("inf"), device="cuda")
    gate[::2] = -float("inf")
    X[1] = 0.0
    R[1] = 0.0
    X[2, 5] = float("nan")
    Y, H = sn.sn_block_norm(X, R, gate=gate, gate_fn="sigmoid")
    assert torch.equal(H[0, ::2], R[0, ::2]) and float((H[0, 1::2] - 2.0).abs().max()) < 1e-5
    assert float(H[1].abs().max()) == 0.0 and float(Y[1].abs().max()) == 0.0
    assert bool(Y[2].isnan().all()) and bool(Y[3].isfinite().all())


def test_no_rows():
    X = torch.zeros(0, 16, device="cuda")
    Y, H = sn.sn_block_norm(X, X, torch.ones(16, device="cuda"), gate=X)
    assert Y.shape == H.shape == (0, 16)
    gw = torch.ones(16, device="cuda")
    dX, dR, dg = sn.sn_block_norm_backward(X, X, X, gate=X, gw=gw)
    assert dX.shape == dR.shape == dg.shape == (0, 16) and float(gw.min()) == 1.0
