"""Limits and refusals of the block norm, the gated feed-forward block and the orthogonalised
updates that no GPU is needed for."""
import pytest

import paper_2506_01260_amd as sn
from test_abi_more_operators import P, _mats, _orth


@pytest.mark.parametrize("steps,code", [(1, 0), (8, 0), (9, 2), (16, 2)])
def test_orthogonalising_steps(steps, code):
    """Behind 8 steps what float32 rounds away fills directions that the matrix lacks."""
    empty = (None, 0, 60, 60, 1)
    assert _orth([empty], [empty], steps=steps) == code
    st = sn.lib().sn_muon_step(1, _mats(empty), _mats(empty), _mats((None, 0, 60, 60, 0)), 0.1, 0.9, 1, 0.0, 1.0,
                               steps, P[15], 1 << 30, None)
    assert st == code
