"""Limits and refusals of the block norm, the gated feed-forward block and the orthogonalised
updates that no GPU is needed for."""
import pytest
import torch

import paper_2506_01260_amd as sn
from test_abi_more_operators import BLOCK, BLOCK_BASE, BLOCK_BWD, P, _call, _mats, _orth


@pytest.mark.parametrize("steps,code", [(1, 0), (8, 0), (9, 2), (16, 2)])
def test_orthogonalising_steps(steps, code):
    """Behind 8 steps what float32 rounds away fills directions that the matrix lacks."""
    empty = (None, 0, 60, 60, 1)
    assert _orth([empty], [empty], steps=steps) == code
    st = sn.lib().sn_muon_step(1, _mats(empty), _mats(empty), _mats((None, 0, 60, 60, 0)), 0.1, 0.9, 1, 0.0, 1.0,
                               steps, P[15], 1 << 30, None)
    assert st == code


def test_missing_operands():
    """What a call cannot do without is refused by name, not by an attribute of None."""
    x = torch.zeros(4, 8)
    calls = {
        "X": [lambda: sn.sn_block_norm(None, x), lambda: sn.sn_block_norm_backward(None, x, x),
              lambda: sn.sn_gated_ff(None, x, x), lambda: sn.sn_gated_ff_backward(None, x, x, x, x, x)],
        "residual": [lambda: sn.sn_block_norm(x, None)],
        "H": [lambda: sn.sn_block_norm_backward(x, None, x)],
        "Wg": [lambda: sn.sn_gated_ff(x, None, x), lambda: sn.sn_gated_ff_backward(x, None, x, x, x, x)],
        "Wu": [lambda: sn.sn_gated_ff(x, x, None), lambda: sn.sn_gated_ff_backward(x, x, None, x, x, x)],
        "G": [lambda: sn.sn_gated_ff_backward(x, x, x, None, x, x), lambda: sn.sn_muon_step([x], None, [x], 0.1),
              lambda: sn.sn_muon_step(x, None, x, 0.1)],
        "U": [lambda: sn.sn_gated_ff_backward(x, x, x, x, None, x)],
        "dH": [lambda: sn.sn_gated_ff_backward(x, x, x, x, x, None)],
        "mats": [lambda: sn.sn_orthogonalize(None), lambda: sn.sn_orthogonalize([x, None])],
        "W": [lambda: sn.sn_muon_step(None, [x], [x], 0.1), lambda: sn.sn_muon_step([None], [x], [x], 0.1)],
        "M": [lambda: sn.sn_muon_step([x], [x], None, 0.1), lambda: sn.sn_muon_step([x], [x], [None], 0.1)],
    }
    for name, group in calls.items():
        for k, call in enumerate(group):
            with pytest.raises(sn.SnError) as e:
                call()
            assert e.value.status == 1 and f"{name}" in str(e.value), (name, k, str(e.value))


def test_gains_without_the_post_norm_are_not_looked_at():
    """w_post is read only with the post norm: without it any pointer goes, whatever its alignment.
    (Each call is refused for another reason, behind that check, so that nothing runs.)"""
    fwd = dict(BLOCK_BASE, post=0, w_post=P[2] + 1)
    assert _call("sn_block_norm", BLOCK, fwd, dict(Y=P[5])) == 5
    assert _call("sn_block_norm", BLOCK, fwd, dict(Y=P[5], post=1)) == 4
    bwd = {k: v for k, v in fwd.items() if k not in ("R", "ldr", "H", "ldh", "Y", "ldy")}
    bwd.update(H=P[1], ldh=300, dY=P[5], lddy=300, dH=P[6], lddh=300, dX=P[7], lddx=300, dR=P[8], lddr=300,
               dgate=None, lddgate=0, dgate_row=None, gw=P[9], gw_post=None, ws=None, ws_bytes=0)
    assert _call("sn_block_norm_backward", BLOCK_BWD, bwd, {}) == 1
    assert _call("sn_block_norm_backward", BLOCK_BWD, bwd, dict(post=1)) == 4
