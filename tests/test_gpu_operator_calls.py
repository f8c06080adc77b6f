"""The binding's two forms of the calls on logits, norms and gradients (native and
Python) give the same bits, on every argument form; and row counts past 2^20, where
the grid has a second dimension."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import logprobs, rmsnorm

pytestmark = pytest.mark.gpu


def _bits(out):
    ts = out if isinstance(out, tuple) else (out,)
    return [None if t is None else t.clone().contiguous().view(torch.uint8) for t in ts]


def _calls(dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def rand(*shape, dt=dtype):
        return torch.randn(shape, generator=g, device="cuda").to(dt)

    n, v, d = 37, 999, 300
    Z, X, R, w = rand(n, v + 5)[:, :v], rand(n, d + 3)[:, :d], rand(n, d), rand(d)
    one = rand(2, 70001)  # few long rows: a workspace
    tok = torch.randint(-1, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    wt = torch.rand(n, generator=g, device="cuda")
    r = sn.sn_token_logprobs(Z, tok)
    f32 = torch.float32
    yield "logprobs", lambda: sn.sn_token_logprobs(Z, tok, n_top=4, scale=0.5)
    yield "logprobs, no tokens", lambda: sn.sn_token_logprobs(Z, scale=2)
    yield "logprobs in parts", lambda: sn.sn_token_logprobs(one, n_top=3)
    yield "backward", lambda: sn.sn_token_logprobs_backward(Z, r.stats, r.entropy, tok, wt, wt)
    yield "backward in place", lambda: (lambda c: sn.sn_token_logprobs_backward(
        c, r.stats, tok=tok, g_logp=wt, out=c))(Z.clone())
    yield "loss", lambda: sn.sn_token_loss(Z, tok, weight=wt, scale=0.5)
    yield "loss, no weights", lambda: sn.sn_token_loss(Z, tok, out=torch.empty_like(Z))
    yield "norm", lambda: sn.sn_rmsnorm(X, w, residual=R)
    yield "norm, plain", lambda: sn.sn_rmsnorm(X)
    yield "norm, in place", lambda: (lambda x: sn.sn_rmsnorm(x, w, residual=R, resid_out=x))(X.clone())
    yield "quant", lambda: sn.sn_rmsnorm_quant(X, w, residual=R, group=128)
    yield "quant, rows", lambda: sn.sn_rmsnorm_quant(X, w, eps=1e-5)

    def backward(**kw):
        gw = torch.ones(d, device="cuda")
        return sn.sn_rmsnorm_backward(X, R, w, gw=gw, **kw), gw

    yield "norm backward", lambda: backward(dH=R)
    ws = torch.empty(sn.sn_rmsnorm_backward_workspace_bytes(n, d, sn._dt(X)), dtype=torch.uint8,
                     device="cuda")
    yield "norm backward, workspace", lambda: backward(workspace=ws)
    yield "norm backward, frozen gains", lambda: sn.sn_rmsnorm_backward(X, R, w)
    grads = [rand(40, 50), rand(7, dt=f32), rand(3, 4, 5), rand(0, 4)]
    total = sn.sn_grad_sumsq(grads)
    yield "sumsq", lambda: sn.sn_grad_sumsq(grads)

    def clip(inside):
        own = [t.clone() for t in grads]
        out = None if inside else [torch.zeros_like(t) for t in grads]
        norm = sn.sn_grad_clip(own, total, 1.0, out=out)
        return (norm, *(own if inside else out))

    yield "clip", lambda: clip(True)
    yield "clip into others", lambda: clip(False)


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

    spy = Spy()
    for name, call in _calls(dtype):
        taken.clear()
        monkeypatch.setattr(sn, "_native", lambda: spy)
        a = _bits(call())
        assert taken and all(taken), f"{name}: the native form stepped aside"
        monkeypatch.setattr(sn, "_native", lambda: None)
        b = _bits(call())
        monkeypatch.undo()
        assert len(a) == len(b), name
        for x, y in zip(a, b):
            assert (x is None) == (y is None) and (x is None or torch.equal(x, y)), name


def test_views_that_the_native_form_leaves():
    """Strided gradients and another stream go through the Python form."""
    g = torch.randn(30, 40, device="cuda")
    s = sn.sn_grad_sumsq([g[:, :30]])
    assert abs(float(s) - float(g[:, :30].double().square().sum())) < 1e-9 * float(s)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    t = sn.sn_grad_sumsq([g[:, :30]], stream=st)
    st.synchronize()
    assert torch.equal(s, t)


def test_more_than_2_20_rows():
    log("[2^20 rows]")
    n, v = (1 << 20) + 77, 9
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    Z = torch.randn(n, v, generator=g, device="cuda")
    tok = torch.randint(0, v, (n,), generator=g, device="cuda", dtype=torch.int32)
    pick = list(range(5)) + list(range((1 << 20) - 3, (1 << 20) + 5)) + list(range(n - 5, n))
    r = sn.sn_token_logprobs(Z, tok, n_top=2)
    zh, th = host(Z[pick]), tok[pick].cpu().numpy()
    ref = logprobs.token_logprobs(zh, th, 2)
    assert np.abs(host(r.logp[pick]) - ref[0]).max() < 1e-5
    assert np.array_equal(r.top_id[pick].cpu().numpy(), ref[4])
    _, dZ = sn.sn_token_loss(Z, tok)
    assert np.abs(host(dZ[pick]) - logprobs.token_loss(zh, th)[1]).max() < 1e-5
    dZ = sn.sn_token_logprobs_backward(Z, r.stats, r.entropy, tok, r.logp, r.logp)
    gl = ref[0]
    assert np.abs(host(dZ[pick]) - logprobs.token_logprobs_backward(zh, th, gl, gl)).max() < 1e-5
    n = (1 << 22) + 77  # four rows to a workgroup
    X = torch.randn(n, 8, generator=g, device="cuda")
    pick = list(range(5)) + list(range((1 << 22) - 3, (1 << 22) + 5)) + list(range(n - 5, n))
    Y, _ = sn.sn_rmsnorm(X)
    assert np.abs(host(Y[pick]) - rmsnorm.rmsnorm(host(X[pick]))[0]).max() < 1e-5
    gw = torch.zeros(8, device="cuda")
    dX = sn.sn_rmsnorm_backward(X, Y, gw=gw)
    ref, _ = rmsnorm.rmsnorm_backward(host(X[pick]), host(Y[pick]))
    assert np.abs(host(dX[pick]) - ref).max() < 1e-5
    want = float((Y[:, 3].double().square()).sum())  # dy h rho = y^2 where dy = y, w = 1
    assert abs(float(gw[3]) - want) < 1e-4 * want
