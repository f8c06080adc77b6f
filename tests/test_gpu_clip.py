"""GPU parity of the gradient norm and clipping through the binding against the
float64 oracle.

Tolerances: the sum of squares is float64, of exact products: 2^-53 for each of
the additions a value passes (at most 512 + 2^10), so 1e-12; the norm is rounded
once to float32; a product g f carries f's rounding and its own, 2^-23 of it, and
for bf16 half an ulp more, 2^-8.
"""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2506_01260_amd as sn
from gpu_helpers import host, log
from oracle import clip as orc

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _grads(seed, shapes, dtypes, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g) * std).to(DT[dtypes[i % len(dtypes)]]).cuda()
            for i, s in enumerate(shapes)]


def _sets():
    yield "one value", [(1,)], ["f32"]
    yield "odd vectors", [(k,) for k in (1, 2, 3, 7, 8, 9, 2047, 2048, 2049, 16384, 16385)], ["bf16", "f32"]
    yield "a small model", [(256, 256), (256,), (1024, 256), (256, 1024)] * 4 + [(1024, 256)], ["f32"]
    yield "many tensors", [(33,)] * 300 + [(5, 77)] * 70, ["bf16", "f32"]
    yield "empty among them", [(0,), (5, 0), (40, 3), (0, 4), (3,)], ["f32", "bf16"]
    yield "three axes", [(4, 5, 6), (2, 3, 4, 5)], ["bf16"]
    yield "large units", [(4096, 2500), (131,)], ["bf16"]


@pytest.mark.parametrize("clips", [True, False])
@pytest.mark.parametrize("name,shapes,dtypes", list(_sets()))
def test_matches_oracle(name, shapes, dtypes, clips):
    log(f"[clip] {name} clips={clips}")
    grads = _grads(len(shapes), shapes, dtypes)
    before = [host(g) for g in grads]
    total = orc.sumsq(before)
    got = sn.sn_grad_sumsq(grads)
    assert got.dtype == torch.float64 and got.shape == (1,)
    assert abs(float(got) - total) <= 1e-12 * total
    most = math.sqrt(total) * (0.3 if clips else 1.5)
    norm, want = orc.clip(before, float(got), most)
    outs = [torch.empty_like(g) for g in grads]
    n1 = sn.sn_grad_clip(grads, got, most, out=outs)
    assert abs(float(n1) - norm) <= 2.0 ** -23 * norm and n1.dtype == torch.float32
    for g, b in zip(grads, before):
        assert np.array_equal(host(g), b)
    n2 = sn.sn_grad_clip(grads, got, most)
    assert torch.equal(n1, n2)
    for g, o, ref in zip(grads, outs, want):
        assert torch.equal(g, o)
        tol = (2.0 ** -23 + (2.0 ** -8 if g.dtype == torch.bfloat16 else 0)) * np.abs(ref)
        assert (np.abs(host(o) - ref) <= tol + 1e-37).all()
        if not clips:
            assert np.array_equal(host(o), ref)


def test_strides_and_odd_starts():
    """Matrices with gaps between rows, columns of a matrix, views that start at odd
    elements, transposed tensors without gaps refused as they are."""
    log("[clip strides]")
    base = _grads(1, [(40, 300), (5000,), (70, 9), (3, 20000)], ["bf16", "f32"])
    for pick in (lambda b: [b[0][:, 1:200], b[1][1:4098], b[2][:, 2], b[3][:, 7:19001]],
                 lambda b: [b[0][::2], b[1][::3], b[2][1:, :5]]):
        bs = [b.clone() for b in base]
        grads = pick(bs)
        before = [host(g) for g in grads]
        total = orc.sumsq(before)
        s = sn.sn_grad_sumsq(grads)
        assert abs(float(s) - total) <= 1e-12 * total
        most = 0.4 * math.sqrt(total)
        _, want = orc.clip(before, float(s), most)
        outs = [torch.empty(g.shape, dtype=g.dtype, device="cuda") for g in grads]
        sn.sn_grad_clip(grads, s, most, out=outs)
        sn.sn_grad_clip(grads, s, most)
        for g, o, ref in zip(grads, outs, want):
            assert torch.equal(g, o)
            assert (np.abs(host(o) - ref) <= 2.0 ** -8 * np.abs(ref) + 1e-37).all()
        # what lies between is untouched
        marked = [torch.ones_like(b, dtype=torch.bool) for b in bs]
        for m in pick(marked):
            m.fill_(False)
        for b, b0, m in zip(bs, base, marked):
            assert torch.equal(b[m], b0[m])


@pytest.mark.parametrize("count,gaps", [(64, 1), (65, 1), (128, 0), (129, 0), (200, 200), (257, 3)])
def test_many_tensors_with_and_without_gaps(count, gaps):
    """Both forms of the table of tensors, at and past its ends."""
    log(f"[clip many tensors] {count}, {gaps} of them with gaps")
    grads = _grads(count, [(3 + i % 5, 20 + 31 * i % 700) for i in range(count)], ["bf16", "f32"])
    for i in range(gaps):
        grads[-1 - i] = grads[-1 - i][:, 1:]
    before = [host(g) for g in grads]
    total = orc.sumsq(before)
    got = sn.sn_grad_sumsq(grads)
    assert abs(float(got) - total) <= 1e-12 * total
    _, want = orc.clip(before, float(got), 0.5 * math.sqrt(total))
    outs = [torch.empty_like(g) for g in grads]
    sn.sn_grad_clip(grads, got, 0.5 * math.sqrt(total), out=outs)
    sn.sn_grad_clip(grads, got, 0.5 * math.sqrt(total))
    for g, o, ref in zip(grads, outs, want):
        assert torch.equal(g, o)
        tol = (2.0 ** -23 + (2.0 ** -8 if g.dtype == torch.bfloat16 else 0)) * np.abs(ref)
        assert (np.abs(host(o) - ref) <= tol + 1e-37).all()


def test_extreme_values():
    log("[clip extremes]")
    inf, nan = float("inf"), float("nan")
    for dtype in ("f32", "bf16"):
        g = _grads(2, [(1000,), (50,)], [dtype], std=1e30)  # squares overflow a float
        before = [host(x) for x in g]
        total = orc.sumsq(before)
        s = sn.sn_grad_sumsq(g)
        assert abs(float(s) - total) <= 1e-12 * total
        n = sn.sn_grad_clip(g, s, 1.0)
        assert abs(float(n) - math.sqrt(total)) <= 2.0 ** -23 * math.sqrt(total)
        left = math.sqrt(orc.sumsq([host(x) for x in g]))
        assert abs(left - 1) < 2.0 ** -8
        # an infinite norm gives 0 and NaN, a NaN norm NaN; +inf never scales
        g = _grads(3, [(100,), (100,)], [dtype])
        keep = [x.clone() for x in g]
        g[0][7] = inf
        s = sn.sn_grad_sumsq(g)
        assert float(s) == inf
        out = [torch.empty_like(x) for x in g]
        assert float(sn.sn_grad_clip(g, s, 1.0, out=out)) == inf
        assert math.isnan(float(out[0][7])) and float(out[1].abs().max()) == 0.0
        g[0][7] = nan
        s = sn.sn_grad_sumsq(g)
        sn.sn_grad_clip(g, s, inf)
        assert math.isnan(float(s)) and all(bool(torch.isnan(x).all()) for x in g)
        s = sn.sn_grad_sumsq(keep)
        mine = [x.clone() for x in keep]
        sn.sn_grad_clip(mine, s, inf)
        assert all(torch.equal(a, b) for a, b in zip(mine, keep))
        sn.sn_grad_clip(mine, s, 0.0)
        assert all(float(a.abs().max()) == 0.0 for a in mine)
    zero = [torch.zeros(300, device="cuda")]
    s = sn.sn_grad_sumsq(zero)
    assert float(s) == 0.0 and float(sn.sn_grad_clip(zero, s, 1.0)) == 0.0
    assert float(zero[0].abs().max()) == 0.0


def test_two_ranks_sums_add():
    """Each half's sum, added, clips like the whole."""
    log("[clip halves]")
    g = _grads(4, [(3000,), (77, 50)], ["f32"])
    whole = sn.sn_grad_sumsq(g)
    both = sn.sn_grad_sumsq(g[:1]) + sn.sn_grad_sumsq(g[1:])
    assert abs(float(whole) - float(both)) <= 1e-12 * float(whole)
    out = torch.empty(1, dtype=torch.float64, device="cuda")
    assert sn.sn_grad_sumsq(g, out=out) is out and torch.equal(out, whole)


def test_more_than_2_31_elements():
    log("[clip 2^31]")
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-1], g[n // 2] = 3.0, 4.0
    s = sn.sn_grad_sumsq([g])
    assert float(s) == 25.0
    assert float(sn.sn_grad_clip([g], s, 2.5)) == 5.0
    assert float(g[-1]) == 1.5 and float(g[n // 2]) == 2.0


def test_refusals_streams_and_none():
    log("[clip refusals]")
    g = _grads(5, [(64, 32), (100,)], ["bf16", "f32"])
    s = sn.sn_grad_sumsq(g)
    flat = torch.zeros(200, device="cuda")
    for status, call in (
            (2, lambda: sn.sn_grad_sumsq([g[0].cpu()])),
            (3, lambda: sn.sn_grad_sumsq([g[0].half()])),
            (2, lambda: sn.sn_grad_sumsq([torch.zeros(1, 64, device="cuda").expand(16, 64)])),
            (2, lambda: sn.sn_grad_sumsq([torch.zeros(4, 5, 6, device="cuda").transpose(0, 2)])),
            (2, lambda: sn.sn_grad_sumsq(g, out=torch.zeros(1, device="cuda"))),
            (9, lambda: sn.sn_grad_sumsq(g, workspace=torch.zeros(4, dtype=torch.uint8, device="cuda"))),
            (2, lambda: sn.sn_grad_clip(g, s, -1.0)),
            (2, lambda: sn.sn_grad_clip(g, s, float("nan"))),
            (2, lambda: sn.sn_grad_clip(g, s.float(), 1.0)),
            (2, lambda: sn.sn_grad_clip(g, s, 1.0, out=g[:1])),
            (2, lambda: sn.sn_grad_clip(g, s, 1.0, out=[g[0], g[1][:50]])),
            (3, lambda: sn.sn_grad_clip(g, s, 1.0, out=[g[0], g[1].bfloat16()])),
            (5, lambda: sn.sn_grad_clip([g[0], g[0]], s, 1.0)),
            (5, lambda: sn.sn_grad_clip([flat[:100]], s, 1.0, out=[flat[50:150]])),
            (5, lambda: sn.sn_grad_clip([flat[:100], flat[100:]], s, 1.0, out=[flat[100:], flat[:100]]))):
        with pytest.raises(sn.SnError) as e:
            call()
        assert e.value.status == status, e.value
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out = [torch.empty_like(x) for x in g]
    t = sn.sn_grad_sumsq(g, stream=st)
    n = sn.sn_grad_clip(g, t, 1.0, out=out, stream=st)
    st.synchronize()
    assert torch.equal(t, s)
    assert torch.equal(n, sn.sn_grad_clip(g, s, 1.0))
    assert all(torch.equal(a, b) for a, b in zip(g, out))
    none = sn.sn_grad_sumsq([])
    assert float(none) == 0.0 and float(sn.sn_grad_clip([], none, 1.0)) == 0.0
    empty = [torch.zeros(0, device="cuda")]
    assert float(sn.sn_grad_clip(empty, sn.sn_grad_sumsq(empty), 1.0)) == 0.0


def test_deterministic_and_in_a_graph():
    log("[clip graph]")
    g = _grads(6, [(513, 257), (100,), (70, 70)] * 30, ["bf16", "f32"])
    out = [torch.empty_like(x) for x in g]
    keep = {}

    def step():
        keep["s"] = sn.sn_grad_sumsq(g)
        keep["n"] = sn.sn_grad_clip(g, keep["s"], 1.0, out=out)

    step()
    want = [t.clone() for t in (keep["s"], keep["n"], *out)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in (keep["s"], keep["n"], *out):
            t.fill_(3)
        sn.sn_grad_sumsq(g[:2])
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(want, (keep["s"], keep["n"], *out)):
            assert torch.equal(x, y)
