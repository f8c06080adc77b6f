"""A block's feed-forward half as it is used: norm, gated feed-forward, down projection, the block's
end with the next norm, backward through all of it and the orthogonalised update of its weights.
Gradients against automatic differentiation, replays of a captured graph against eager calls, other
streams, and the binding's two forms."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log

pytestmark = pytest.mark.gpu

ALPHA, LR = 0.75, 0.02


class Half:
    """Parameters and one training step of the half-block; the loss is sum(Y cY) + sum(H cH)."""

    def __init__(self, n, d, ff, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)

        def rand(*shape, std=1.0, mean=0.0):
            return (torch.randn(shape, generator=g) * std + mean).to(dtype).cuda()
        self.X, self.cY, self.cH = rand(n, d), rand(n, d, std=0.1), rand(n, d, std=0.1)
        self.p = {"w0": rand(d, std=0.1, mean=1.0), "Wg": rand(d, ff, std=d ** -0.5),
                  "Wu": rand(d, ff, std=d ** -0.5), "W2": rand(d, ff, std=ff ** -0.5),
                  "wp": rand(d, std=0.1, mean=1.0), "gate": rand(d), "w1": rand(d, std=0.1, mean=1.0)}
        self.M = {n_: torch.zeros(self.p[n_].shape, device="cuda") for n_ in ("Wg", "Wu", "W2")}

    def forward_backward(self):
        p = self.p
        Y0, _ = sn.sn_rmsnorm(self.X, p["w0"])
        A, G, U = sn.sn_gated_ff(Y0, p["Wg"], p["Wu"], save=True)
        O = A @ p["W2"].t()
        kw = dict(w_post=p["wp"], gate=p["gate"], gate_fn="sigmoid", alpha=ALPHA)
        Y, H = sn.sn_block_norm(O, self.X, p["w1"], **kw)
        g = {n_: torch.zeros(p[n_].shape, device="cuda") for n_ in ("w0", "wp", "gate", "w1")}
        dO, dX, _ = sn.sn_block_norm_backward(O, H, self.cY, p["w1"], dH=self.cH, gw=g["w1"],
                                              gw_post=g["wp"], dgate=g["gate"], **kw)
        g["W2"] = dO.t() @ A
        dY0, g["Wg"], g["Wu"] = sn.sn_gated_ff_backward(Y0, p["Wg"], p["Wu"], G, U, dO @ p["W2"])
        g["X"] = sn.sn_rmsnorm_backward(self.X, dY0, p["w0"], dH=dX, gw=g["w0"])
        return Y, H, g

    def update(self, g):
        p, M = self.p, self.M
        sn.sn_muon_step([p["Wg"], p["Wu"]], [g["Wg"], g["Wu"]], [M["Wg"], M["Wu"]], LR)
        sn.sn_muon_step([p["W2"]], [g["W2"]], [M["W2"]], LR, weight_decay=1e-3)

    def state(self):
        return [*self.p.values(), *self.M.values()]


def test_gradients_against_differentiation():
    """float32: within 1e-5 of each gradient's norm, some ten roundings of 2^-24 over sums of up to
    300 terms in five layers."""
    log("[half block gradients]")
    torch.backends.cuda.matmul.allow_tf32 = False
    m = Half(70, 96, 130, torch.float32, 1)
    Y, H, g = m.forward_backward()
    p = {k: v.double().cpu().requires_grad_() for k, v in {**m.p, "X": m.X}.items()}

    def norm(x, w):
        return x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-6) * w
    y0 = norm(p["X"], p["w0"])
    a = torch.nn.functional.silu(y0 @ p["Wg"]) * (y0 @ p["Wu"])
    h = ALPHA * p["X"] + torch.sigmoid(p["gate"]) * norm(a @ p["W2"].t(), p["wp"])
    y = norm(h, p["w1"])
    ((y * m.cY.double().cpu()).sum() + (h * m.cH.double().cpu()).sum()).backward()
    assert float((Y.cpu() - y.detach()).abs().max()) < 1e-4 and float((H.cpu() - h.detach()).abs().max()) < 1e-4
    for name in sorted(g):
        off = float((g[name].double().cpu() - p[name].grad).norm() / p[name].grad.norm())
        log(f"  {name}: {off:.2e}")
        assert off < 1e-5, name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,d,ff", [(5, 64, 136), (200, 96, 250)])
def test_graph_replays_match_eager(dtype, n, d, ff):
    """Two training steps captured together; every replay from the same start gives the eager steps'
    bits, with eager work on the same tensors between the replays."""
    log(f"[half block graph] {dtype} {n} {d} {ff}")
    eager, m = Half(n, d, ff, dtype), Half(n, d, ff, dtype)
    start = [t.clone() for t in m.state()]

    def two(x):
        for _ in range(2):
            Y, H, g = x.forward_backward()
            x.update(g)
        return Y, H, g
    want_out = two(eager)
    want = [t.clone() for t in eager.state()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):  # warm up where the products allocate
        two(m)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = two(m)
    for replay in range(4):
        for t, s in zip(m.state(), start):
            t.copy_(s)
        for t in (out[0], out[1], *out[2].values()):
            t.fill_(float("nan"))
        Half(7, 32, 40, dtype, replay).forward_backward()  # eager work of the program's own
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(m.state(), want)), replay
        assert torch.equal(out[0], want_out[0]) and torch.equal(out[1], want_out[1])
        assert all(torch.equal(out[2][k], want_out[2][k]) for k in out[2])


def test_two_streams_at_once():
    """The same calls on two streams, given by argument, do not disturb each other."""
    log("[half block streams]")
    X = [torch.randn(300, 128, device="cuda").bfloat16() for _ in range(2)]
    Wg, Wu = (torch.randn(128, 520, device="cuda").bfloat16() * 0.1 for _ in range(2))
    R = [torch.randn(300, 128, device="cuda").bfloat16() for _ in range(2)]
    mats = [[torch.randn(90, 130, device="cuda") for _ in range(3)] for _ in range(2)]

    def calls(i, stream):
        H, G, U = sn.sn_gated_ff(X[i], Wg, Wu, save=True, stream=stream)
        grads = sn.sn_gated_ff_backward(X[i], Wg, Wu, G, U, H, stream=stream)
        Y, S = sn.sn_block_norm(X[i], R[i], stream=stream)
        with torch.cuda.stream(stream):  # None: the current one
            gw = torch.zeros(128, device="cuda")
        back = sn.sn_block_norm_backward(X[i], S, Y, gw=gw, stream=stream)
        return [H, *grads, Y, S, *back[:2], gw, *sn.sn_orthogonalize(mats[i], stream=stream)]
    want = [calls(i, None) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [calls(i, s) for i, s in enumerate(streams)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def _calls(dtype):
    g = torch.Generator().manual_seed(3)

    def rand(*shape, dt=dtype):
        return torch.randn(shape, generator=g).to(dt).cuda()
    n, d, ff = 37, 300, 136
    X, R, w, row, tok = rand(n, d + 4)[:, :d], rand(n, d), rand(d), rand(d), rand(n, d)
    yield "block norm", lambda: sn.sn_block_norm(X, R, w, w_post=w, gate=row, gate_fn="sigmoid", alpha=2)
    yield "block norm, plain", lambda: sn.sn_block_norm(X, R, post=False)
    yield "block norm, in place", lambda: (lambda r: sn.sn_block_norm(X, r, w, gate=tok, resid_out=r))(R.clone())

    def back(gate, **kw):
        gw, gw1 = torch.ones(d, device="cuda"), torch.ones(d, device="cuda")
        return (*sn.sn_block_norm_backward(X, R, tok, w, w_post=w, gate=gate, gw=gw, gw_post=gw1, **kw), gw, gw1)
    yield "block norm backward, row", lambda: back(row, dH=R, dgate=torch.ones(d, device="cuda"))
    yield "block norm backward, token", lambda: back(tok, gate_fn="sigmoid")
    ws = torch.empty(sn.sn_block_norm_backward_workspace_bytes(n, d, sn._dt(X)), dtype=torch.uint8, device="cuda")
    yield "block norm backward, workspace", lambda: back(None, workspace=ws)
    yield "block norm backward, frozen", lambda: sn.sn_block_norm_backward(X, R, None, post=False, dH=tok)
    Wg, Wu, G, U, dH = rand(d, ff), rand(d, ff), rand(n, ff), rand(n, ff), rand(n, ff)
    one = rand(1, d)
    yield "gated ff", lambda: sn.sn_gated_ff(X, Wg, Wu)
    yield "gated ff, one token", lambda: sn.sn_gated_ff(one, Wg, Wu, act="gelu", save=True)
    yield "gated ff, given", lambda: sn.sn_gated_ff(X, Wg, Wu, act="relu", out=torch.empty_like(G),
                                                   out_g=torch.empty_like(G), out_u=torch.empty_like(G))
    yield "gated ff backward", lambda: sn.sn_gated_ff_backward(X, Wg, Wu, G, U, dH)
    yield "gated ff backward, dX", lambda: sn.sn_gated_ff_backward(X, Wg, Wu, G, U, dH, want_gw=False)[0]

    def added():
        w = torch.ones(2, d, ff, device="cuda")
        return sn.sn_gated_ff_backward(X, Wg, Wu, G, U, dH, dG=torch.empty_like(G), dU=torch.empty_like(G),
                                       gWg=w[0], gWu=w[1], accumulate=True)
    yield "gated ff backward, added", added
    mats = [rand(40, 70) for _ in range(3)]
    yield "orthogonalize", lambda: tuple(sn.sn_orthogonalize(mats, steps=3))
    yield "orthogonalize, in place", lambda: (lambda c: tuple(sn.sn_orthogonalize(c, out=c)))([m.clone() for m in mats])

    def muon():
        W, M = [m.clone() for m in mats], [torch.ones(40, 70, device="cuda") for _ in mats]
        assert sn.sn_muon_step(W, mats, M, 0.1, nesterov=False) is W
        return (*W, *M)
    yield "muon", muon


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_native_and_python_forms_agree(dtype, monkeypatch):
    log(f"[binding forms] {dtype}")
    sn.lib()
    taken = []

    class Spy:
        def __getattr__(self, name):
            f = getattr(sn._bound, name)

            def call(*a):
                r = f(*a)
                taken.append(r is not None)
                return r
            return call

    def bits(out):
        ts = out if isinstance(out, tuple) else (out,)
        return [None if t is None else t.clone().contiguous().view(torch.uint8) for t in ts]
    spy = Spy()
    for name, call in _calls(dtype):
        taken.clear()
        monkeypatch.setattr(sn, "_native", lambda: spy)
        a = bits(call())
        assert taken and all(taken), f"{name}: the native form stepped aside"
        monkeypatch.setattr(sn, "_native", lambda: None)
        b = bits(call())
        monkeypatch.undo()
        assert len(a) == len(b), name
        for x, y in zip(a, b):
            assert (x is None) == (y is None) and (x is None or torch.equal(x, y)), name


def test_refusals_of_the_binding():
    X, w, g = torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    W = torch.zeros(8, 16, device="cuda")
    H = torch.zeros(4, 16, device="cuda")
    for call, status in (
            (lambda: sn.sn_block_norm(X, None), 1), (lambda: sn.sn_block_norm(X, X.bfloat16()), 3),
            (lambda: sn.sn_block_norm(X, X[:3]), 2), (lambda: sn.sn_block_norm(X, X, w[:7]), 2),
            (lambda: sn.sn_block_norm(X, X, gate=w[:7]), 2), (lambda: sn.sn_block_norm(X, X, gate=X[:3]), 2),
            (lambda: sn.sn_block_norm(X, X, gate=w.bfloat16()), 3),
            (lambda: sn.sn_block_norm(X, X, resid_out=X, out=X), 5),
            (lambda: sn.sn_block_norm_backward(X, X, X, gw_post=g, post=False), 1),
            (lambda: sn.sn_block_norm_backward(X, X, None, gw=g), 1),
            (lambda: sn.sn_block_norm_backward(X, X, X, dgate=g), 2),
            (lambda: sn.sn_block_norm_backward(X, X, X, gate=X, dgate=g), 2),
            (lambda: sn.sn_gated_ff(X, W, W[:, :8]), 2), (lambda: sn.sn_gated_ff(X, W.bfloat16(), W), 3),
            (lambda: sn.sn_gated_ff(X, W[:7], W[:7]), 2),
            (lambda: sn.sn_gated_ff(X, W, torch.zeros(8, 20, device="cuda")[:, :16]), 2),
            (lambda: sn.sn_gated_ff(X, W, W, out=W[:4]), 5),
            (lambda: sn.sn_gated_ff(X.t().contiguous().t(), W, W), 2),
            (lambda: sn.sn_gated_ff_backward(X, W, W, H, H, H[:, :8]), 2),
            (lambda: sn.sn_gated_ff_backward(X, W, W, H, H, H, gWg=W.half(), gWu=W.half()), 3),
            (lambda: sn.sn_gated_ff_backward(X, W, W, H, H, H, workspace=torch.zeros(1, device="cuda")), 9),
            (lambda: sn.sn_orthogonalize([W, X]), 2), (lambda: sn.sn_orthogonalize([W], steps=0), 2),
            (lambda: sn.sn_orthogonalize([W], out=[]), 2), (lambda: sn.sn_orthogonalize(W.half()), 3),
            (lambda: sn.sn_muon_step([W], [W], [], 0.1), 2), (lambda: sn.sn_muon_step([W], [W], [W], 0.1), 5)):
        with pytest.raises(sn.SnError) as e:
            call()
        assert e.value.status == status, str(e.value)
    assert np.isfinite(host(W)).all()
