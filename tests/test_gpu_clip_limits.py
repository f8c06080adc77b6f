"""Gradient norm and clipping at their limits: blocks of one matrix as separate
tensors."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import clip as orc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_column_blocks_in_place(dtype):
    """The parts of a fused gradient beside ordinary tensors: the norm's list is also the
    clipping's, in place and into blocks of another matrix, and what belongs to no block
    stays (tolerances as in test_gpu_clip.py)."""
    log(f"[clip blocks] {dtype}")
    g = torch.Generator().manual_seed(3)
    whole = torch.randn(50, 1001, generator=g).to(dtype).cuda()
    plain = torch.randn(5000, generator=g).to(dtype).cuda()
    cuts = ((0, 333), (333, 334), (334, 700), (701, 1001))  # column 700 belongs to none

    def parts(m):
        return [m[:, a:b] for a, b in cuts] + [plain if m is whole else torch.empty_like(plain)]

    grads = parts(whole)
    before, kept = [host(x) for x in grads], whole[:, 700].clone()
    total = orc.sumsq(before)
    s = sn.sn_grad_sumsq(grads)
    assert abs(float(s) - total) <= 1e-12 * total
    most = 0.25 * math.sqrt(total)
    _, want = orc.clip(before, float(s), most)
    other = torch.full((50, 1003), 7.0, dtype=dtype, device="cuda")
    outs = parts(other)
    sn.sn_grad_clip(grads, s, most, out=outs)
    sn.sn_grad_clip(grads, s, most)
    for x, o, ref in zip(grads, outs, want):
        assert torch.equal(x, o)
        tol = (2.0 ** -23 + (2.0 ** -8 if dtype == torch.bfloat16 else 0)) * np.abs(ref)
        assert (np.abs(host(o) - ref) <= tol + 1e-37).all()
    assert torch.equal(whole[:, 700], kept)
    assert bool((other[:, 700] == 7).all()) and bool((other[:, 1001:] == 7).all())
    with pytest.raises(sn.SnError) as e:
        sn.sn_grad_clip([whole[:, :333], whole[:, 332:400]], s, most)
    assert e.value.status == 5


def test_more_units_than_a_grid_dimension_has():
    """Units of 256 threads past 2^24, so past 2^32 threads of one launch.  The norm: one
    matrix of 2^18 + 1 rows with gaps, a row a unit, listed 64 times.  Clipping: 2^24 + 99
    rows of 4097, again a row a unit; of its memory the first and last rows are looked at."""
    log("[clip units past 2^24]")
    if torch.cuda.mem_get_info()[0] < 160e9:
        pytest.skip("needs 140 GB of device memory")
    rows, cols = (1 << 18) + 1, 32769
    g = torch.zeros(rows, cols + 1, dtype=torch.bfloat16, device="cuda")
    g[0, 0], g[-1, cols - 1], g[:, cols] = 3.0, 4.0, float("nan")
    s = sn.sn_grad_sumsq([g[:, :cols]] * 64)
    assert float(s) == 64 * 25.0
    del g
    torch.cuda.empty_cache()
    rows, cols = (1 << 24) + 99, 4097
    g = torch.empty(rows, cols + 1, dtype=torch.bfloat16, device="cuda")
    for part in (g[:5], g[-5:], g[(1 << 24) - 3:(1 << 24) + 3]):
        part.fill_(6.0)
    norm = sn.sn_grad_clip([g[:, :cols]], torch.full((1,), 16.0, dtype=torch.float64, device="cuda"), 2.0)
    assert float(norm) == 4.0
    for part in (g[:5], g[-5:], g[(1 << 24) - 3:(1 << 24) + 3]):
        assert bool((part[:, :cols] == 3.0).all()) and bool((part[:, cols] == 6.0).all())
    del g, part
    torch.cuda.empty_cache()
