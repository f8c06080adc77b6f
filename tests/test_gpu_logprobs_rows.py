"""Log probabilities of more than 512 rows, where workgroups of 256, 512 and 1024
threads take the rows: special rows among ordinary ones, odd widths (so that bf16
rows start at odd elements), against the float64 oracle.  Tolerances are those of
test_gpu_logprobs.py."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
import test_gpu_logprobs as base
from gpu_helpers import host, log
from oracle import logprobs as orc

pytestmark = pytest.mark.gpu

INF = float("inf")
# (dtype, width, alternatives): more than 1024 pieces of 8 bf16 or 4 floats.  Without
# alternatives 512 threads below 7168 pieces and 1024 from there on; with them 256
# threads up to 4096 pieces and 512 above.
CASES = [(dt, e * p + 1, n_top) for dt, e in (("bf16", 8), ("f32", 4))
         for p, n_top in ((1025, 0), (5000, 0), (7166, 0), (7167, 0), (1024, 5), (1024, 64), (4095, 1),
                          (4095, 33), (4096, 5), (5000, 17), (5000, 64), (7168, 32))]


def _only(r, allowed):
    keep = r[list(allowed)].clone()
    r.fill_(-INF)
    r[list(allowed)] = keep


def _special(Z):
    """Fills rows among the others; returns their numbers."""
    v, low = Z.shape[1], torch.finfo(Z.dtype).min
    j = torch.arange(v).to(Z.device)
    fills = [
        lambda r: r.fill_(1.5),                       # all equal
        lambda r: r.copy_(torch.round(r)),            # many ties
        lambda r: r[1:].fill_(-INF),                  # one allowed
        lambda r: r.fill_(-INF),                      # none
        lambda r: r.fill_(low),
        lambda r: r[::2].fill_(low),
        lambda r: r[::3].fill_(-INF),
        lambda r: r.copy_(j.flip(0) / 512.0),         # descending, ties in bf16
        lambda r: r.copy_(j / 512.0),                 # ascending
        lambda r: (r.fill_(-0.0), r[::2].fill_(0.0)),
        lambda r: _only(r, range(0, 3)),              # few allowed, together and apart
        lambda r: _only(r, range(v // 2, v // 2 + 20)),
        lambda r: _only(r, range(v - 30, v)),
        lambda r: _only(r, range(7, v, v // 15)),
        lambda r: _only(r, range(0, v, v // 300)),
        lambda r: r.copy_(r > 0),                     # few values
        lambda r: r.copy_(torch.clamp(torch.round(r), -20, 3)),
        lambda r: r.copy_(j % 2 + j // 300 % 3),
        lambda r: r[:700].add_(100.0),                # large ones in one place
        lambda r: r[v - 700:].add_(100.0),
        lambda r: (r.copy_(-300.0 - r.abs()), r[v // 3:].fill_(-300.0)),
        lambda r: r[v - 1].fill_(float("nan")),       # no distribution
        lambda r: r[0].fill_(-float("nan")),
        lambda r: r[v // 2].fill_(INF),
    ]
    rows = list(range(3, len(Z) - 6, 17))[:len(fills)]
    assert len(rows) == len(fills)
    for i, fill in zip(rows, fills):
        fill(Z[i])
    return rows


@pytest.mark.parametrize("dtype,v,n_top", CASES)
def test_special_rows_among_many(dtype, v, n_top):
    log(f"[logprobs many long rows] {dtype} V={v} top {n_top}")
    n, scale = 521, 0.9
    Z = base._logits(v + n_top, n, v, dtype).contiguous()
    pick = _special(Z)
    pick = sorted(set(pick + [0, 1, 2, 4, 255, 256, 511, 512, 513, n - 1] + [p + 1 for p in pick[::4]]))
    tok = base._tokens(v, n, v)
    tok[pick[::3]] = v - 1
    r = sn.sn_token_logprobs(Z, torch.tensor(tok, dtype=torch.int32).cuda(), n_top=n_top, scale=scale)
    zh, tk = host(Z[pick]), tok[pick]
    logp, H, stats, top_logp, top_id = orc.token_logprobs(zh, tk, n_top, scale)
    lp = orc.log_p(zh, scale)
    ax, s, L, a, x2 = base._bounds(zh, lp, scale)
    axt = np.where(tk >= 0, ax[np.arange(len(pick)), np.maximum(tk, 0)], 0)
    base._near(host(r.logp[pick]), logp, base.U * (4 + 2 * axt + 2 * L + s), "logp")
    base._near(host(r.entropy[pick]), H, base.U * (4 + 2 * L + s * (1 + a) + 4 * x2), "entropy")
    base._near(host(r.stats[pick][:, 0]), stats[:, 0], 0.0, "stats m")
    base._near(host(r.stats[pick][:, 1]), stats[:, 1], base.U * (4 + 2 * L + s), "stats L")
    if n_top:
        assert np.array_equal(r.top_id[pick].cpu().numpy(), top_id)
        axj = np.take_along_axis(ax, np.maximum(top_id, 0), 1)
        base._near(host(r.top_logp[pick]), top_logp, base.U * (4 + 2 * axj + (2 * L + s)[:, None]), "top")
    again = sn.sn_token_logprobs(Z, torch.tensor(tok, dtype=torch.int32).cuda(), n_top=n_top, scale=scale)
    for x, y in zip(r, again):  # the same bits, NaN rows too
        assert x is y or torch.equal(x.view(torch.int32), y.view(torch.int32))


@pytest.mark.parametrize("v", [1025, 1500, 2047, 2048])
def test_backward_with_two_waves_to_a_float32_row(v):
    base.test_backward_matches_oracle("f32", 6, v)
