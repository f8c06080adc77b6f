"""The norm's row layouts that the widths of test_gpu_rmsnorm.py leave out: both sides
of 768 and 1536 pieces of 8 bf16 or 4 floats, and the backward's larger and odd numbers
of workgroups."""
from __future__ import annotations

import pytest

import test_gpu_rmsnorm as base
from paper_2506_01260_amd import sn_rmsnorm_backward_workspace_bytes

pytestmark = pytest.mark.gpu

# (float32 rows of exactly 768 pieces are left out)
WIDTHS = [("bf16", d) for d in (6136, 6143, 6144, 6145, 12280, 12287, 12288, 12289)] + \
         [("f32", d) for d in (3068, 3071, 3073, 3076, 6140, 6143, 6144, 6145)]


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_forward(dtype, d):
    base.test_forward_matches_oracle(dtype, d)


@pytest.mark.parametrize("dtype,d", WIDTHS)
def test_backward(dtype, d):
    base.test_backward_matches_oracle(dtype, d)


@pytest.mark.parametrize("n,d,groups", [(8201, 1001, 1024), (8200, 2055, 1024), (6151, 5003, 768),
                                        (4099, 6201, 512), (6143, 5003, 768)])
def test_backward_of_many_rows(n, d, groups):
    """Rows of an odd number of bf16 values: 1024 workgroups of four rows; with a row to a
    workgroup one fewer than `groups`, which is even, from 8 rows to each on (the last
    case has fewer)."""
    assert sn_rmsnorm_backward_workspace_bytes(n, d, 1) == -(-4 * groups * d // 256) * 256
    base.test_backward_of_many_odd_rows(n, d)
