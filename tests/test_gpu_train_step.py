"""The example's training step: its gradients against automatic differentiation of
the same model in float64 on the CPU, its clipping, and that it learns."""
from __future__ import annotations

import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import log

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                    "train_step.py")


def _example():
    spec = importlib.util.spec_from_file_location("train_step", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _autograd(model, tok, target, weight):
    """(logp, gradients) of the same model by torch's differentiation, float64, CPU."""
    p = {n: w.detach().double().cpu().requires_grad_() for n, w in model.p.items()}
    U, E, P = (t.double().cpu() for t in (model.U, model.E, model.P))
    tok, target, weight = tok.long().cpu(), target.long().cpu(), weight.double().cpu()
    table = E[tok] + P[torch.arange(len(tok)) % model.seq]

    def norm(h, g):
        return h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * g

    X0 = table + p["CS"][tok] @ U.t()
    X1 = X0 + torch.relu(norm(X0, p["g1"]) @ p["W1"]) @ p["W2"].t()
    X2 = X1 + torch.relu(norm(X1, p["g2"]) @ p["W3"]) @ p["W4"].t()
    Xr = (X2 - table) @ U @ U.t() + table
    logp = torch.log_softmax(norm(Xr, p["g3"]) @ p["Wo"].t(), 1)
    logp = torch.where(target >= 0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    (-(weight * logp).sum()).backward()
    return logp.detach(), {n: w.grad for n, w in p.items()}


def test_gradients_against_differentiation():
    """float32: every gradient within 1e-4 of its norm (the products alone, in
    float32 over up to 1024 terms and seven layers deep, are good to about 1e-5)."""
    log("[train step gradients]")
    ex = _example()
    torch.backends.cuda.matmul.allow_tf32 = False
    model = ex.Model(torch.float32, seed=3, vocab=200, d=96, k=12, ff=130, seq=24)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    tok, target = ex.batch(g, n_seq=3, seq=24, vocab=200)
    weight = torch.rand(len(tok), generator=g, device="cuda")
    logp, grads = model.gradients(tok, target, weight)
    ref_logp, ref = _autograd(model, tok, target, weight)
    assert float((logp.cpu().double() - ref_logp).abs().max()) < 1e-4
    assert set(grads) == set(ref)
    for n in sorted(ref):
        off = float((grads[n].cpu().double() - ref[n]).norm() / ref[n].norm())
        log(f"  {n}: {off:.2e}")
        assert off < 1e-4, n
    # the clipped gradients' norm, and the steps that the optimizer takes with them
    total = sum(float(r.square().sum()) for r in ref.values()) ** 0.5
    before = {n: w.clone() for n, w in model.p.items()}
    norm = model.update(grads, lr=1e-3, max_norm=0.25 * total)
    assert abs(float(norm) - total) < 1e-4 * total
    left = float(sn.sn_grad_sumsq([grads[n] for n in grads])) ** 0.5
    assert abs(left - 0.25 * total) < 1e-4 * total
    assert all(not torch.equal(before[n], w) for n, w in model.p.items())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_it_learns(dtype):
    log(f"[train step {dtype}]")
    losses, right = _example().main(steps=60, dtype=dtype, log=log)
    assert np.isfinite(losses).all()
    assert losses[-1] < 0.5 * losses[0], losses
    assert right >= 0.75  # the next token is a function of the present one
    log(f"  {losses[0]:.3f} -> {losses[-1]:.3f}, {right:.0%} of the answers right")
