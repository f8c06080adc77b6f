"""Training steps of a small language model cut into two pipeline stages, both on
this GPU, with every step around the matrix products in the library's kernels:

    stage 1   token table -> norm -> MLP -> norm (residual added) -> MLP -> compress
    stage 2   decompress -> norm -> output matrix -> loss and its gradient
    and back  norm backward -> gradient codec -> ... -> token table's gradient
    update    global norm, clipping, (modified) AdamW

The task is synthetic: the next token is a fixed function of the present one.

    python examples/train_step.py [--steps 40] [--dtype bf16]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_01260_amd as sn  # noqa: E402

VOCAB, D, K, FF, BATCH, SEQ = 1024, 256, 32, 512, 8, 128


class Model:
    """The two stages' parameters, gradients and optimizer state."""

    def __init__(self, dtype=torch.bfloat16, seed=0, vocab=VOCAB, d=D, k=K, ff=FF, seq=SEQ):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rand(*shape, std):
            return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

        self.dtype, self.seq = dtype, seq
        self.U = torch.linalg.qr(torch.randn(d, k, generator=g, device="cuda"))[0].to(dtype).contiguous()
        self.basis = sn.sn_basis_pack(self.U)
        self.E, self.P = rand(vocab, d, std=0.5), rand(seq, d, std=0.1)  # fixed tables
        self.CS = sn.sn_grad_compress(self.basis, self.E)                # T_S = T_fixed U U^T
        self.p = {
            "CS": self.CS,
            "g1": torch.ones(d, dtype=dtype, device="cuda"),
            "W1": rand(d, ff, std=d ** -0.5), "W2": rand(d, ff, std=0.5 * ff ** -0.5),
            "g2": torch.ones(d, dtype=dtype, device="cuda"),
            "W3": rand(d, ff, std=d ** -0.5), "W4": rand(d, ff, std=0.5 * ff ** -0.5),
            "g3": torch.ones(d, dtype=dtype, device="cuda"),
            "Wo": rand(vocab, d, std=d ** -0.5),
        }
        # W2 and W4 are stored [out, in]; their columns start, and stay, in the subspace
        sn.sn_project_weights_multi(self.basis, [self.p["W2"], self.p["W4"]])
        self.M = {n: torch.zeros(self._mat(w).shape, device="cuda") for n, w in self.p.items()}
        self.V = {n: torch.zeros_like(m) for n, m in self.M.items()}
        self.t = 0

    @staticmethod
    def _mat(w):
        return w if w.dim() == 2 else w[None]

    def gradients(self, tok, target, weight=None):
        """(log probabilities of the targets, gradients) of one micro-batch; tok and
        target: int32 vectors of whole sequences, target -1 where there is none."""
        p, b = self.p, self.basis
        tables = dict(tok=tok, E=self.E, P=self.P, seq_len=self.seq)
        if weight is None:
            weight = torch.full((len(tok),), 1.0 / max(1, int((target >= 0).sum())), device="cuda")
        # stage 1
        X0 = sn.sn_embed_lowrank_forward(b, p["CS"], tok, E=self.E, P=self.P, seq_len=self.seq)
        Y1, _ = sn.sn_rmsnorm(X0, p["g1"])
        A1 = torch.relu(Y1 @ p["W1"])
        O1 = A1 @ p["W2"].t()
        Y2, X1 = sn.sn_rmsnorm(O1, p["g2"], residual=X0)
        A2 = torch.relu(Y2 @ p["W3"])
        X2 = X1 + A2 @ p["W4"].t()
        # the boundary, and stage 2
        Xr = sn.sn_decompress(b, sn.sn_compress(b, X2, **tables), **tables)
        Y3, _ = sn.sn_rmsnorm(Xr, p["g3"])
        logits = Y3 @ p["Wo"].t()
        logp, dZ = sn.sn_token_loss(logits, target, weight=weight, out=logits)
        g = {n: torch.zeros(p[n].shape, device="cuda") for n in ("g1", "g2", "g3", "CS")}
        g["Wo"] = dZ.t() @ Y3
        dXr = sn.sn_rmsnorm_backward(Xr, dZ @ p["Wo"], p["g3"], gw=g["g3"])
        # the boundary again, and back through stage 1
        dX2 = sn.sn_decompress(b, sn.sn_grad_compress(b, dXr))
        g["W4"] = dX2.t() @ A2
        dU = (dX2 @ p["W4"]) * (A2 > 0)
        g["W3"] = Y2.t() @ dU
        dX1 = sn.sn_rmsnorm_backward(X1, dU @ p["W3"].t(), p["g2"], dH=dX2, gw=g["g2"])
        g["W2"] = dX1.t() @ A1
        dU = (dX1 @ p["W2"]) * (A1 > 0)
        g["W1"] = Y1.t() @ dU
        dX0 = sn.sn_rmsnorm_backward(X0, dU @ p["W1"].t(), p["g1"], dH=dX1, gw=g["g1"])
        sn.sn_embed_lowrank_backward(b, dX0, tok, g["CS"])
        return logp, g

    def update(self, g, lr, max_norm=1.0):
        """Clip the gradients to max_norm and take one AdamW step; returns the norm."""
        names = sorted(g)
        # with the stages on GPUs of their own, total is summed over them here
        total = sn.sn_grad_sumsq([g[n] for n in names])
        norm = sn.sn_grad_clip([g[n] for n in names], total, max_norm)
        self.t += 1
        for n in names:
            w = self._mat(self.p[n])
            sn.sn_adamw_step(w, self._mat(g[n]).to(w.dtype), self.M[n], self.V[n], self.t, lr,
                             subspace=n in ("W2", "W4"))
        # inside a stage gradients leave the subspace: back to it, so that the boundary
        # stays without loss
        sn.sn_project_weights_multi(self.basis, [self.p["W2"], self.p["W4"]])
        return norm

    def answer(self, tok, n_top=3):
        """The tokens most likely to follow the last of each sequence, with their log
        probabilities; the last norm's output in 8 bits, as an 8-bit product takes it."""
        p, b = self.p, self.basis
        X0 = sn.sn_embed_lowrank_forward(b, p["CS"], tok, E=self.E, P=self.P, seq_len=self.seq)
        A = torch.relu(sn.sn_rmsnorm(X0, p["g1"])[0] @ p["W1"])
        Y, X = sn.sn_rmsnorm(A @ p["W2"].t(), p["g2"], residual=X0)
        X += torch.relu(Y @ p["W3"]) @ p["W4"].t()
        last = X[self.seq - 1::self.seq]
        Q, S, _ = sn.sn_rmsnorm_quant(last, p["g3"])
        logits = ((Q.to(self.dtype) @ p["Wo"].t()) * S).to(self.dtype)
        r = sn.sn_token_logprobs(logits, n_top=n_top)
        return r.top_id, r.top_logp


def batch(g, n_seq=BATCH, seq=SEQ, vocab=VOCAB):
    """Random sequences, and for each token t the one to answer with, 5 t + 7; a
    sequence's first position has none, as padding has none."""
    tok = torch.randint(0, vocab, (n_seq, seq), generator=g, device="cuda", dtype=torch.int32)
    target = (5 * tok + 7) % vocab
    target[:, 0] = -1
    return tok.reshape(-1), target.reshape(-1)


def main(steps=40, dtype="bf16", lr=1e-2, log=print):
    model = Model(torch.bfloat16 if dtype == "bf16" else torch.float32)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    losses = []
    for step in range(steps):
        tok, target = batch(g)
        logp, grads = model.gradients(tok, target)
        norm = model.update(grads, lr)
        losses.append(-float(logp.sum()) / int((target >= 0).sum()))
        if step % 10 == 0 or step == steps - 1:
            log(f"step {step}: loss {losses[-1]:.4f}, gradient norm {float(norm):.4f}")
    tok, target = batch(g)
    ids, lp = model.answer(tok)
    want = target[SEQ - 1::SEQ]
    log(f"answers: {ids[:, 0].tolist()} (wanted {want.tolist()}), "
        f"probabilities {[round(math.exp(v), 3) for v in lp[:, 0].tolist()]}")
    return losses, float((ids[:, 0] == want).float().mean())


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    main(a.steps, a.dtype)
