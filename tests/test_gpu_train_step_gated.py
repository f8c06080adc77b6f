"""The example's training step with gated blocks and orthogonalised updates: it runs, its gradients
against automatic differentiation of the same model in float64 on the CPU, and W2's and W4's columns
in the subspace after an update."""
from __future__ import annotations

import importlib.util
import math
import os

import pytest
import torch

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
    p = {n: w.detach().double().cpu().requires_grad_() for n, w in model.p.items()}
    U, E, P = (t.double().cpu() for t in (model.U, model.E, model.P))
    tok, target, weight = tok.long().cpu(), target.long().cpu(), weight.double().cpu()
    table = E[tok] + P[torch.arange(len(tok)) % model.seq]

    def norm(h, g=1.0):
        return h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * g

    def block(x, g, wg, wu, w2):
        y = norm(x, p[g])
        return x + norm((torch.nn.functional.silu(y @ p[wg]) * (y @ p[wu])) @ p[w2].t())

    X2 = block(block(table + p["CS"][tok] @ U.t(), "g1", "W1", "V1", "W2"), "g2", "W3", "V3", "W4")
    Xr = (X2 - table) @ U @ U.t() + table
    logp = torch.log_softmax(norm(Xr, p["g3"]) @ p["Wo"].t(), 1)
    logp = torch.where(target >= 0, logp.gather(1, target.clamp(min=0)[:, None])[:, 0], 0.0)
    (-(weight * logp).sum()).backward()
    return logp.detach(), {n: w.grad for n, w in p.items()}


def test_gradients_against_differentiation():
    """float32: every gradient within 1e-4 of its norm (products in float32 over up to 1024 terms and
    nine layers deep are good to about 1e-5)."""
    log("[gated train step gradients]")
    ex = _example()
    torch.backends.cuda.matmul.allow_tf32 = False
    model = ex.GatedModel(torch.float32, seed=3, vocab=200, d=96, k=12, ff=130, seq=24)
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
    # an update takes every parameter along, and W2 and W4 not out of the subspace: their part
    # outside is that of a projection's float32 roundings, 2^-24 times some sums of 96 terms
    before = {n: w.clone() for n, w in model.p.items()}
    model.update(grads, lr=1e-2)
    assert all(not torch.equal(before[n], w) for n, w in model.p.items())
    U = model.U.double()
    for n in ("W2", "W4"):
        w = model.p[n].double()
        assert float((w - U @ (U.t() @ w)).norm() / w.norm()) < 1e-5, n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_it_runs(dtype):
    log(f"[gated train step {dtype}]")
    losses, _ = _example().main(steps=6, dtype=dtype, log=log, gated=True)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses)
