"""Host-side argument checks of the block norm, the gated feed-forward block and the
orthogonalised updates (no GPU): each call fails validation or has nothing to do, so nothing
touches a device.  The same file runs against the library whose host code is built under
AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2506_01260_amd as sn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = [0x7F0000000000 + (i << 24) for i in range(16)]
NAN, INF = float("nan"), float("inf")
BIG = 1 << 31


def _call(name, order, base, over):
    a = dict(base)
    a.update(over)
    assert set(a) == set(order.split()), set(a) ^ set(order.split())
    st = getattr(sn.lib(), name)(*[a[k] for k in order.split()])
    if st:
        assert sn.lib().sn_last_error().decode() != ""
    return st


BLOCK = "X N d ldx dt R ldr post w_post gate ldgate fn alpha w eps H ldh Y ldy stream"
BLOCK_BASE = dict(X=P[0], N=8, d=300, ldx=300, dt=1, R=P[1], ldr=300, post=1, w_post=P[2], gate=P[3],
                  ldgate=0, fn=0, alpha=1.0, w=P[4], eps=1e-6, H=P[5], ldh=300, Y=P[6], ldy=300,
                  stream=None)


@pytest.mark.parametrize("over,code", [
    (dict(dt=4), 3), (dict(N=-1), 2), (dict(N=BIG), 2), (dict(d=0), 2), (dict(ldx=299), 2),
    (dict(ldr=1), 2), (dict(ldh=299), 2), (dict(ldy=299), 2), (dict(ldgate=299), 2), (dict(fn=2), 8),
    (dict(fn=-1), 8), (dict(alpha=NAN), 2), (dict(alpha=INF), 2), (dict(eps=-1.0), 2),
    (dict(eps=NAN), 2), (dict(X=None), 1), (dict(R=None), 1), (dict(H=None), 1), (dict(X=P[0] + 1), 4),
    (dict(w=P[4] + 1), 4), (dict(w_post=P[2] + 1), 4), (dict(gate=P[3] + 1), 4), (dict(R=P[1] + 1), 4),
    (dict(H=P[5] + 1), 4), (dict(Y=P[6] + 1), 4), (dict(dt=0, X=P[0] + 2), 4), (dict(Y=P[0]), 5),
    (dict(Y=P[5]), 5), (dict(H=P[0] + 2), 5), (dict(H=P[1], ldh=301), 5), (dict(H=P[2]), 5),
    (dict(H=P[3] + 100), 5), (dict(Y=P[3] - 200, ldgate=300), 5), (dict(Y=P[4]), 5),
    (dict(N=0, X=None, R=None, H=None), 0)])
def test_block_norm(over, code):
    assert _call("sn_block_norm", BLOCK, BLOCK_BASE, over) == code


BLOCK_BWD = ("X N d ldx dt H ldh post w_post gate ldgate fn alpha w eps dY lddy dH lddh dX lddx dR lddr "
             "dgate lddgate dgate_row gw gw_post ws ws_bytes stream")


@pytest.mark.parametrize("over,code", [
    (dict(dt=7), 3), (dict(d=0), 2), (dict(lddy=1), 2), (dict(lddh=1), 2), (dict(lddx=299), 2),
    (dict(lddr=299), 2), (dict(fn=3), 8), (dict(eps=INF), 2), (dict(dX=None), 1), (dict(dR=None), 1),
    (dict(H=None), 1), (dict(dY=None), 1), (dict(post=0), 1), (dict(dgate=P[12], lddgate=300), 2),
    (dict(gate=None), 2), (dict(ldgate=300), 2), (dict(ldgate=300, dgate_row=None, dgate=P[12], lddgate=9), 2),
    (dict(dY=P[5] + 1), 4), (dict(gw=P[9] + 2), 4), (dict(gw_post=P[10] + 1), 4),
    (dict(dgate_row=P[11] + 2), 4), (dict(dX=P[1]), 5), (dict(dX=P[8]), 5), (dict(dX=P[2]), 5),
    (dict(dR=P[0]), 5), (dict(dX=P[0], lddx=301), 5), (dict(gw=P[10]), 5), (dict(dgate_row=P[9] + 400), 5),
    (dict(dX=P[3]), 5), (dict(ws=None), 1), (dict(ws=P[12] + 8), 4), (dict(ws_bytes=100), 9),
    (dict(ws=P[7] - 256), 5), (dict(N=0, X=None, H=None, dX=None, dR=None), 0)])
def test_block_norm_backward(over, code):
    base = {k: v for k, v in BLOCK_BASE.items() if k not in ("R", "ldr", "H", "ldh", "Y", "ldy")}
    base.update(H=P[1], ldh=300, dY=P[5], lddy=300, dH=P[6], lddh=300, dX=P[7], lddx=300, dR=P[8],
                lddr=300, dgate=None, lddgate=0, dgate_row=P[11], gw=P[9], gw_post=P[10], ws=P[12],
                ws_bytes=1 << 22)
    assert _call("sn_block_norm_backward", BLOCK_BWD, base, over) == code


def test_block_norm_workspace():
    f = sn.sn_block_norm_backward_workspace_bytes
    assert f(8, 300, 1) >= 3 * 300 * 4 and f(100000, 4096, 1) >= 100 * 4096 * 12
    for bad in ((0, 8, 0), (8, 0, 0), (8, 8, 5), (BIG, 8, 0), (8, BIG, 0)):
        assert f(*bad) == 0


FF = "X N d ldx dt Wg Wu ff ldw act H ldh G U ldg ws ws_bytes stream"
FF_BASE = dict(X=P[0], N=64, d=256, ldx=256, dt=1, Wg=P[1], Wu=P[2], ff=512, ldw=512, act=0, H=P[3],
               ldh=512, G=P[4], U=P[5], ldg=512, ws=P[6], ws_bytes=1 << 24, stream=None)


@pytest.mark.parametrize("over,code", [
    (dict(dt=2), 3), (dict(N=-1), 2), (dict(N=BIG), 2), (dict(d=0, ldx=0), 2), (dict(ff=0), 2),
    (dict(ldx=255), 2), (dict(ldw=511), 2), (dict(ldh=511), 2), (dict(ldg=511), 2), (dict(act=3), 8),
    (dict(act=-1), 8), (dict(X=None), 1), (dict(Wg=None), 1), (dict(Wu=None), 1), (dict(H=None), 1),
    (dict(G=None), 1), (dict(U=None), 1), (dict(X=P[0] + 1), 4), (dict(Wu=P[2] + 1), 4),
    (dict(U=P[5] + 1), 4), (dict(dt=0, Wg=P[1] + 2), 4), (dict(H=P[0]), 5), (dict(H=P[1] + 512), 5),
    (dict(G=P[3]), 5), (dict(U=P[4]), 5), (dict(U=P[4] + 1000), 5), (dict(ldg=1024, U=P[4] + 1022), 5),
    (dict(ldg=1024, G=P[4] + 2, U=P[4] + 1024), 5), (dict(H=P[2]), 5),
    (dict(ldx=257, ws=None), 1), (dict(ldx=257, ws=P[6] + 16), 4), (dict(ldx=257, ws_bytes=64), 9),
    (dict(ldx=257, ws=P[3]), 5), (dict(ldx=257, ws=P[0]), 5),
    (dict(N=1 << 30, d=1 << 12, ldx=1 << 12), 2), (dict(N=0, X=None, H=None), 0)])
def test_gated_ff(over, code):
    assert _call("sn_gated_ff", FF, FF_BASE, over) == code


FF_BWD = ("X N d ldx dt Wg Wu ff ldw act G U ldg dH lddh dG dU ldd dX lddx gWg gWu ldgw gdt acc ws "
          "ws_bytes stream")
FF_BWD_BASE = dict(X=P[0], N=64, d=256, ldx=256, dt=1, Wg=P[1], Wu=P[2], ff=512, ldw=512, act=0, G=P[3],
                   U=P[4], ldg=512, dH=P[5], lddh=512, dG=P[6], dU=P[7], ldd=512, dX=P[8], lddx=256,
                   gWg=P[9], gWu=P[10], ldgw=512, gdt=1, acc=0, ws=P[11], ws_bytes=1 << 24, stream=None)


@pytest.mark.parametrize("over,code", [
    (dict(dt=2), 3), (dict(gdt=2), 3), (dict(dt=0, gdt=1), 3), (dict(N=BIG), 2), (dict(ldg=511), 2),
    (dict(lddh=511), 2), (dict(ldd=511), 2), (dict(lddx=255), 2), (dict(ldgw=511), 2), (dict(act=9), 8),
    (dict(X=None), 1), (dict(G=None), 1), (dict(dH=None), 1), (dict(dG=None), 1), (dict(gWg=None), 1),
    (dict(gWu=None), 1), (dict(dH=P[5] + 1), 4), (dict(gdt=0, gWg=P[9] + 2), 4), (dict(dX=P[8] + 1), 4),
    (dict(dX=P[0]), 5), (dict(dX=P[6]), 5), (dict(dG=P[0]), 5), (dict(dG=P[3] + 2), 5),
    (dict(dG=P[3], ldd=513), 5), (dict(dU=P[6]), 5), (dict(gWu=P[9] + 512), 5), (dict(gWg=P[1]), 5),
    (dict(ldgw=1024, gWu=P[9] + 1022), 5), (dict(ldx=257, ws=None), 1),
    (dict(ldx=257, ws_bytes=10), 9), (dict(ldx=257, ws=P[7]), 5), (dict(ldx=257, ws=P[8] - 256), 5), (dict(N=0, acc=1, X=None, G=None), 0),
    (dict(N=0, gWg=None, gWu=None), 0)])
def test_gated_ff_backward(over, code):
    # a row stride that is no multiple of 8 needs a workspace
    assert _call("sn_gated_ff_backward", FF_BWD, FF_BWD_BASE, over) == code


@pytest.mark.parametrize("dt", [0, 1])
def test_gated_ff_workspace(dt):
    f, b = sn.sn_gated_ff_workspace_bytes, sn.sn_gated_ff_backward_workspace_bytes
    if dt == 1:
        assert f(32768, 4096, 14336, 4096, 14336, dt, True) == 0
        assert b(32768, 4096, 14336, 4096, 14336, 14336, dt, True) == 0
    whole = 32768 * 4096 * 2
    assert f(32768, 4096, 14336, 4096, 14336, dt, False) >= whole
    assert f(32768, 4095, 14336, 4096, 14336, dt, True) >= whole
    assert b(32768, 4096, 14336, 4100, 14336, 14336, dt, True) >= whole
    for bad in ((0, 8, 8, 8, 8, dt, True), (8, 0, 8, 8, 8, dt, True), (8, 8, 0, 8, 8, dt, True),
                (8, 8, 8, 7, 8, dt, True), (8, 8, 8, 8, 7, dt, True), (8, 8, 8, 8, 8, 2, True),
                (BIG, 8, 8, 8, 8, dt, True)):
        assert f(*bad) == 0
        assert b(*bad[:5], 8, *bad[5:]) == 0
    assert b(64, 256, 512, 256, 512, 511, dt, True) == 0


def _mats(*specs):
    return (sn._Tensor * max(1, len(specs)))(*[sn._Tensor(*s) for s in specs])


def _orth(src, dst, steps=5, ws=P[15], ws_bytes=1 << 30, count=None):
    st = sn.lib().sn_orthogonalize(len(src) if count is None else count, _mats(*src) if src else None,
                                   _mats(*dst) if dst else None, steps, ws, ws_bytes, None)
    if st:
        assert sn.lib().sn_last_error().decode() != ""
    return st


def test_orthogonalize():
    a, b = (P[0], 40, 60, 60, 1), (P[1], 40, 60, 60, 1)
    assert _orth([], []) == 0 and _orth([a], [b], count=-1) == 2
    assert _orth([], [b], count=1) == 1 and _orth([a], [], count=1) == 1
    for steps in (0, -1, 17):
        assert _orth([a], [b], steps=steps) == 2
    for bad, code in (((None, 40, 60, 60, 1), 1), ((P[0] + 1, 40, 60, 60, 1), 4),
                      ((P[0], 40, 60, 59, 1), 2), ((P[0], 40, 61, 61, 1), 2), ((P[0], 60, 40, 60, 1), 2),
                      ((P[0], 40, 60, 60, 0), 3), ((P[1] + 2, 40, 60, 60, 1), 5), ((P[1], 40, 60, 61, 1), 5)):
        assert _orth([bad], [b]) == code, bad
    assert _orth([a], [(P[0], 40, 60, 60, 2)]) == 3
    assert _orth([(P[0], -1, 60, 60, 1)], [(P[1], -1, 60, 60, 1)]) == 2
    assert _orth([(P[0], 1 << 30, 1 << 12, 1 << 12, 1)], [(P[1], 1 << 30, 1 << 12, 1 << 12, 1)]) == 2
    assert _orth([a, a], [b, b]) == 5                       # the same output twice
    assert _orth([a, (P[2], 40, 60, 60, 1)], [b, a]) == 5   # another's input as output
    assert _orth([a], [b], ws=None) == 1 and _orth([a], [b], ws=P[15] + 8) == 4
    assert _orth([a], [b], ws_bytes=1000) == 9 and _orth([a], [b], ws=P[1]) == 5
    assert _orth([a], [b], ws=P[0] - 512) == 5
    assert _orth([(None, 0, 60, 60, 1)], [(None, 0, 60, 60, 1)]) == 0
    assert _orth([(None, 40, 0, 0, 1)], [(None, 40, 0, 0, 1)]) == 0


def test_orthogonalize_workspace():
    f = sn.sn_orthogonalize_workspace_bytes
    assert f(1, 256, 256) >= 8 * 256 * 256 + 8 * 256 * 256
    assert f(2, 256, 256) > f(1, 256, 256) and f(1000, 256, 256) == f(32, 256, 256)
    for bad in ((0, 8, 8), (-1, 8, 8), (1, 0, 8), (1, 8, 0), (1, BIG, 8), (1, 1 << 30, 1 << 30)):
        assert f(*bad) == 0


@pytest.mark.parametrize("over,code", [
    (dict(lr=-1.0), 2), (dict(lr=NAN), 2), (dict(lr=INF), 2), (dict(momentum=1.0), 2),
    (dict(momentum=-0.1), 2), (dict(decay=-1.0), 2), (dict(decay=INF), 2), (dict(scale=NAN), 2),
    (dict(lr=1e30, scale=1e30), 2), (dict(steps=0), 2), (dict(steps=17), 2),
    (dict(W=(P[0], 40, 60, 60, 3)), 3), (dict(G=(P[1], 40, 60, 60, 0)), 3), (dict(M=(P[2], 40, 60, 60, 1)), 3),
    (dict(M=(P[2], 60, 40, 40, 0)), 2), (dict(M=(P[2] + 2, 40, 60, 60, 0)), 4), (dict(M=(None, 40, 60, 60, 0)), 1),
    (dict(G=(P[0], 40, 60, 60, 1)), 5), (dict(M=(P[0], 40, 60, 60, 0)), 5), (dict(M=(P[1] - 4, 40, 60, 60, 0)), 5),
    (dict(ws=P[2]), 5), (dict(ws_bytes=0), 9)])
def test_muon_step(over, code):
    a = dict(W=(P[0], 40, 60, 60, 1), G=(P[1], 40, 60, 60, 1), M=(P[2], 40, 60, 60, 0), lr=0.1, momentum=0.9,
             decay=0.0, scale=1.0, steps=5, ws=P[15], ws_bytes=1 << 30)
    a.update(over)
    st = sn.lib().sn_muon_step(1, _mats(a["W"]), _mats(a["G"]), _mats(a["M"]), a["lr"], a["momentum"], 1,
                               a["decay"], a["scale"], a["steps"], a["ws"], a["ws_bytes"], None)
    assert st == code
    if code:
        assert sn.lib().sn_last_error().decode() != ""


def test_orthogonalize_workspace_covers_every_launch():
    """A call makes its matrices 32 at a time: the bytes of 32 and of what is left, whose fewer
    matrices may be cut into more parts."""
    f = sn.sn_orthogonalize_workspace_bytes
    sizes = [1, 7, 33, 64, 100, 256, 300, 512, 729, 1600, 4267, 20000]
    for rows in sizes:
        for cols in sizes:
            whole = f(32, rows, cols)
            for left in (1, 2, 3, 5, 11, 31):
                assert f(32 + left, rows, cols) == f(64 + left, rows, cols) == max(whole, f(left, rows, cols))


def test_binding_refuses_before_the_library():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    for call, status in (
            (lambda: sn.sn_block_norm(x, x, w, gate_fn="tanh"), 8),
            (lambda: sn.sn_block_norm(x, x, w, next_norm=False, out=x), 2),
            (lambda: sn.sn_gated_ff(x, x, x, act="swish"), 8),
            (lambda: sn.sn_gated_ff(x, x, x, out_g=x), 1),
            (lambda: sn.sn_gated_ff_backward(x, x, x, x, x, x, gWg=x), 1),
            (lambda: sn.sn_gated_ff_backward(x, x, x, x, x, x, accumulate=True), 1)):
        with pytest.raises(sn.SnError) as e:
            call()
        assert e.value.status == status


@pytest.mark.skipif(bool(os.environ.get("SN_LIBRARY")), reason="already running on another build")
def test_under_host_sanitizers():
    from test_abi_hostsan import _asan_runtime
    rt = _asan_runtime()
    if rt is None:
        pytest.skip("g++ with the ASan runtime is not available")
    from paper_2506_01260_amd import build as b
    env = dict(os.environ, SN_LIBRARY=b.build_host_sanitized(), LD_PRELOAD=rt,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider",
                        os.path.abspath(__file__)], cwd=ROOT, env=env, capture_output=True, text=True,
                       timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and " passed" in r.stdout, out[-4000:]
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out[-4000:]
