"""Host-side argument checks of the token log probabilities, the norm and gradient
clipping (no GPU): each call fails validation or has nothing to do, so nothing
touches a device.  The same file runs against the library whose host code is
built under AddressSanitizer and UndefinedBehaviorSanitizer."""
import ctypes
import os
import subprocess
import sys

import pytest

import paper_2506_01260_amd as sn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B, C, D, E, F = (0x7F0000000000 + (i << 24) for i in range(6))
NAN, INF = float("nan"), float("inf")


def _call(name, order, base, over):
    a = dict(base)
    a.update(over)
    assert set(a) == set(order.split()), set(a) ^ set(order.split())
    st = getattr(sn.lib(), name)(*[a[k] for k in order.split()])
    if st:
        assert sn.lib().sn_last_error().decode() != ""
    return st


LOGPROBS = "Z N V ldz dt scale tok logp entropy stats n_top top_logp top_id err ws ws_bytes stream"


@pytest.mark.parametrize("over,code", [
    (dict(dt=2), 3), (dict(N=-1), 2), (dict(N=1 << 31), 2), (dict(V=0), 2), (dict(V=1 << 31), 2),
    (dict(ldz=99), 2), (dict(ldz=1 << 31), 2), (dict(Z=None), 1), (dict(Z=A + 1), 4),
    (dict(tok=B + 2), 4), (dict(logp=None), 1), (dict(entropy=None), 1), (dict(stats=None), 1),
    (dict(stats=E + 2), 4), (dict(n_top=-1), 2), (dict(n_top=101), 2), (dict(n_top=65), 8),
    (dict(n_top=3), 1), (dict(n_top=3, top_logp=F, top_id=F + 8), 5),
    (dict(scale=0.0), 2), (dict(scale=NAN), 2), (dict(scale=INF), 2), (dict(scale=1e-9), 2),
    (dict(entropy=C), 5), (dict(entropy=A + 100), 5), (dict(stats=B + 8), 5),
    (dict(V=100000, ldz=100000), 1), (dict(V=100000, ldz=100000, ws=F + 8), 4),
    (dict(V=100000, ldz=100000, ws=F, ws_bytes=255), 9),
    (dict(V=100000, ldz=100000, ws=A + 256, ws_bytes=1 << 20), 5),
    (dict(V=100000, ldz=100000, ws=D, ws_bytes=1 << 20), 5),
    (dict(N=0, Z=None, logp=None, entropy=None, stats=None), 0)])
def test_logprobs(over, code):
    base = dict(Z=A, N=8, V=100, ldz=100, dt=1, scale=1.0, tok=B, logp=C, entropy=D, stats=E, n_top=0,
                top_logp=None, top_id=None, err=None, ws=None, ws_bytes=0, stream=None)
    assert _call("sn_token_logprobs", LOGPROBS, base, over) == code


def test_logprobs_workspace():
    """Few long rows take a workspace, the rest none; invalid arguments give 0."""
    f = sn.sn_token_logprobs_workspace_bytes
    assert f(1, 128256, 1, 5) > 0 and f(1, 128256, 1, 64) > f(1, 128256, 1, 5) > f(1, 128256, 1, 0)
    assert f(100000, 128256, 1, 5) == 0 and f(1, 1000, 1, 5) == 0
    for bad in ((0, 128256, 1, 5), (1, 0, 1, 0), (1, 128256, 2, 5), (1, 128256, 1, 65), (1, 8, 1, 9),
                (1, 128256, 1, -1), (1 << 31, 128256, 1, 5), (1, 1 << 31, 1, 5)):
        assert f(*bad) == 0


BACKWARD = "Z N V ldz dt scale tok stats entropy g_logp g_entropy dZ lddz err stream"


@pytest.mark.parametrize("over,code", [
    (dict(dt=-1), 3), (dict(V=0, ldz=0), 2), (dict(lddz=99), 2), (dict(Z=None), 1), (dict(dZ=None), 1),
    (dict(stats=None), 1), (dict(tok=None), 1), (dict(g_entropy=F, entropy=None), 1),
    (dict(dZ=F + 1), 4), (dict(g_logp=D + 2), 4), (dict(dZ=A + 2), 5), (dict(dZ=A, lddz=101), 5),
    (dict(dZ=B), 5), (dict(dZ=C - 16), 5), (dict(scale=-1.0), 2), (dict(N=0, Z=None, dZ=None), 0)])
def test_logprobs_backward(over, code):
    base = dict(Z=A, N=8, V=100, ldz=100, dt=1, scale=1.0, tok=B, stats=C, entropy=None, g_logp=D,
                g_entropy=None, dZ=F, lddz=100, err=None, stream=None)
    assert _call("sn_token_logprobs_backward", BACKWARD, base, over) == code


LOSS = "Z N V ldz dt scale tok weight logp dZ lddz err stream"


@pytest.mark.parametrize("over,code", [
    (dict(dt=9), 3), (dict(N=1 << 31), 2), (dict(lddz=1 << 31), 2), (dict(tok=None), 1),
    (dict(logp=None), 1), (dict(dZ=None), 1), (dict(weight=D + 1), 4), (dict(logp=A + 4), 5),
    (dict(logp=A + 4, dZ=A), 5), (dict(logp=B), 5), (dict(dZ=A + 200), 5), (dict(scale=2.0 ** 21), 2),
    (dict(N=0, Z=None, dZ=None, tok=None, logp=None), 0)])
def test_loss(over, code):
    base = dict(Z=A, N=8, V=100, ldz=100, dt=1, scale=1.0, tok=B, weight=None, logp=C, dZ=F, lddz=100,
                err=None, stream=None)
    assert _call("sn_token_loss", LOSS, base, over) == code


NORM = "X N d ldx dt R ldr w eps H ldh Y ldy stream"
NORM_BASE = dict(X=A, N=8, d=300, ldx=300, dt=1, R=B, ldr=300, w=C, eps=1e-6, H=D, ldh=300, Y=E, ldy=300,
                 stream=None)


@pytest.mark.parametrize("over,code", [
    (dict(dt=4), 3), (dict(N=-1), 2), (dict(d=0), 2), (dict(ldx=299), 2), (dict(ldr=1), 2),
    (dict(ldh=299), 2), (dict(ldy=299), 2), (dict(eps=-1.0), 2), (dict(eps=NAN), 2), (dict(eps=INF), 2),
    (dict(X=None), 1), (dict(Y=None), 1), (dict(X=A + 1), 4), (dict(w=C + 1), 4), (dict(Y=E + 1), 4),
    (dict(Y=A), 5), (dict(Y=D), 5), (dict(H=A + 2), 5), (dict(H=A, ldh=301), 5), (dict(H=C), 5),
    (dict(N=0, X=None, Y=None), 0), (dict(N=1 << 31), 2)])
def test_norm(over, code):
    assert _call("sn_rmsnorm", NORM, NORM_BASE, over) == code


QUANT = "X N d ldx dt R ldr w eps H ldh group Q ldq S lds stream"


@pytest.mark.parametrize("over,code", [
    (dict(group=64), 8), (dict(group=-128), 2), (dict(lds=2), 2), (dict(group=0, lds=0), 2),
    (dict(Q=None), 1), (dict(S=None), 1), (dict(S=F + 2), 4), (dict(ldq=299), 2), (dict(Q=F), 5),
    (dict(Q=A + 1000), 5), (dict(dt=3), 3), (dict(N=0, X=None), 0)])
def test_norm_quant(over, code):
    base = {k: v for k, v in NORM_BASE.items() if k not in ("Y", "ldy")}
    base.update(group=128, Q=E, ldq=300, S=F, lds=3)
    assert _call("sn_rmsnorm_quant", QUANT, base, over) == code


NORM_BWD = "H N d ldh dt dY lddy w eps dH lddh dX lddx gw ws ws_bytes stream"


@pytest.mark.parametrize("over,code", [
    (dict(dt=4), 3), (dict(lddy=299), 2), (dict(dH=D + (1 << 20), lddh=299), 2), (dict(lddx=299), 2), (dict(eps=-2.0), 2),
    (dict(H=None), 1), (dict(dY=None), 1), (dict(dX=None), 1), (dict(ws=None), 1), (dict(ws=F + 8), 4),
    (dict(ws_bytes=100), 9), (dict(gw=E + 2), 4), (dict(dX=A), 5), (dict(dX=B + 2), 5),
    (dict(dX=B, lddx=301), 5), (dict(gw=F + 256), 5), (dict(gw=A), 5), (dict(ws=A), 5), (dict(dX=C), 5),
    (dict(N=0, H=None, dY=None, dX=None, ws=None), 0)])
def test_norm_backward(over, code):
    base = dict(H=A, N=8, d=300, ldh=300, dt=1, dY=B, lddy=300, w=C, eps=1e-6, dH=None, lddh=0, dX=D,
                lddx=300, gw=E, ws=F, ws_bytes=1 << 20, stream=None)
    assert _call("sn_rmsnorm_backward", NORM_BWD, base, over) == code


def test_norm_backward_workspace_never_shrinks_with_more_rows():
    for dt in (0, 1):
        for d in (8, 512, 1024, 1025, 4096, 40000):
            last = 0
            for n in list(range(1, 700)) + [4096, 32768, (1 << 31) - 1]:
                need = sn.sn_rmsnorm_backward_workspace_bytes(n, d, dt)
                assert need >= max(last, 4 * d) and need % 256 == 0
                last = need
    assert sn.sn_rmsnorm_backward_workspace_bytes(0, 8, 0) == 0
    assert sn.sn_rmsnorm_backward_workspace_bytes(8, 0, 0) == 0
    assert sn.sn_rmsnorm_backward_workspace_bytes(8, 8, 5) == 0


def _arr(*ts):
    return (sn._Tensor * max(1, len(ts)))(*[sn._Tensor(*t) for t in ts])


G = [(A, 8, 100, 100, 1), (B, 1, 5000, 5000, 0)]


@pytest.mark.parametrize("ts,code", [
    ([(A, 8, 100, 100, 7)], 3), ([(A, -1, 100, 100, 1)], 2), ([(A, 8, -1, 100, 1)], 2),
    ([(A, 8, 100, 99, 1)], 2), ([(A, 8, 100, 1 << 40, 1)], 2), ([(None, 8, 100, 100, 1)], 1),
    ([(A + 1, 8, 100, 100, 1)], 4), ([(A, 1 << 31, 1, 1, 1)], 2), ([(A, 1, 1 << 40, 1, 1)], 2),
    ([(A, 1 << 30, 1 << 30, 1 << 30, 1)], 2), ([(A, 1, 1 << 39, 1, 1)] * 2, 2), ([(E, 8, 4, 4, 0)], 5),
    ([(F - 4, 8, 4, 4, 0)], 5)])
def test_sumsq_refusals(ts, code):
    assert sn.lib().sn_grad_sumsq(len(ts), _arr(*ts), E, F, 1 << 20, None) == code
    if code not in (1, 4, 5):
        assert sn.lib().sn_grad_sumsq_workspace_bytes(len(ts), _arr(*ts)) == 0
    if code != 5:
        assert sn.lib().sn_grad_clip(len(ts), _arr(*ts), None, E, 1.0, F, None) == code


def test_sumsq_arguments():
    L, g = sn.lib(), _arr(*G)
    assert L.sn_grad_sumsq(2, None, E, F, 1 << 20, None) == 1
    assert L.sn_grad_sumsq(-1, g, E, F, 1 << 20, None) == 2
    assert L.sn_grad_sumsq(2, g, None, F, 1 << 20, None) == 1
    assert L.sn_grad_sumsq(2, g, E + 4, F, 1 << 20, None) == 4
    assert L.sn_grad_sumsq(2, g, E, F + 8, 1 << 20, None) == 4
    assert L.sn_grad_sumsq(2, g, E, None, 1 << 20, None) == 1
    need = L.sn_grad_sumsq_workspace_bytes(2, g)
    assert need > 0 and need % 256 == 0
    assert L.sn_grad_sumsq(2, g, E, F, need - 1, None) == 9
    assert L.sn_grad_sumsq(2, g, F + 8, F, need, None) == 5
    assert L.sn_grad_sumsq_workspace_bytes(0, None) > 0


@pytest.mark.parametrize("out,code", [
    ([(C, 8, 99, 99, 1), (D, 1, 5000, 5000, 0)], 2), ([(C, 8, 100, 100, 0), (D, 1, 5000, 5000, 0)], 3),
    ([(C, 8, 100, 98, 1), (D, 1, 5000, 5000, 0)], 2), ([(C, 8, 100, 100, 1), (None, 1, 5000, 5000, 0)], 1),
    ([(C + 1, 8, 100, 100, 1), (D, 1, 5000, 5000, 0)], 4),
    ([(C, 8, 100, 100, 1), (C + 800, 1, 5000, 5000, 0)], 5),        # two outputs
    ([(B + 100, 8, 100, 100, 1), (D, 1, 5000, 5000, 0)], 5),        # another gradient
    ([(A, 8, 100, 101, 1), (D, 1, 5000, 5000, 0)], 5),              # itself, other stride
    ([(A + 2, 8, 100, 100, 1), (B, 1, 5000, 5000, 0)], 5),
    ([(E - 16, 8, 100, 100, 1), (D, 1, 5000, 5000, 0)], 5),         # sumsq
    ([(F, 8, 100, 100, 1), (D, 1, 5000, 5000, 0)], 5)])             # norm
def test_clip_outputs(out, code):
    assert sn.lib().sn_grad_clip(2, _arr(*G), _arr(*out), E, 1.0, F, None) == code


def test_clip_arguments():
    L, g = sn.lib(), _arr(*G)
    assert L.sn_grad_clip(2, g, None, None, 1.0, F, None) == 1
    assert L.sn_grad_clip(2, g, None, E + 4, 1.0, F, None) == 4
    assert L.sn_grad_clip(2, g, None, E, 1.0, F + 2, None) == 4
    assert L.sn_grad_clip(2, g, None, E, -0.5, F, None) == 2
    assert L.sn_grad_clip(2, g, None, E, NAN, F, None) == 2
    assert L.sn_grad_clip(2, g, None, E, 1.0, E + 4, None) == 5
    assert L.sn_grad_clip(2, g, None, A + 8, 1.0, F, None) == 5
    assert L.sn_grad_clip(2, _arr(G[0], G[0]), None, E, 1.0, F, None) == 5
    many = _arr(*[(A + 4096 * i, 1, 1000, 1000, 0) for i in range(3000)], (A + 4096 * 77 + 4, 1, 8, 8, 0))
    assert L.sn_grad_clip(3001, many, None, E, 1.0, F, None) == 5


def test_tensor_struct_matches_the_header():
    assert ctypes.sizeof(sn._Tensor) == 40


def test_under_asan_and_ubsan():
    if os.environ.get("SN_LIBRARY"):
        pytest.skip("this is the run under the sanitizers")
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


def _told_apart(grads, out=None):
    """What the check between tensors says of a list: the call's norm lies over its
    sumsq, which is refused too, after the tensors have been told apart."""
    st = sn.lib().sn_grad_clip(len(grads), _arr(*grads), None if out is None else _arr(*out), E, 1.0,
                               E + 4, None)
    assert st == 5
    return "norm overlaps sumsq" in sn.lib().sn_last_error().decode()


def _slice(r, c, rows, cols, ld, dt, base=A):
    """rows x cols from row r and column c of a matrix of row stride ld."""
    return (base + (r * ld + c) * (2 if dt else 4), rows, cols, ld, dt)


@pytest.mark.parametrize("dt", [0, 1])
def test_clip_tells_column_blocks_apart(dt):
    """Blocks of one matrix (a fused projection's gradient) share no element."""
    def block(*a):
        return _slice(*a, 300, dt)
    assert _told_apart([block(0, 0, 8, 100), block(0, 100, 8, 100), block(0, 200, 8, 100)])
    assert _told_apart([block(0, 200, 8, 100), block(0, 0, 8, 100), block(0, 100, 8, 100)])
    assert _told_apart([block(0, 0, 8, 100), block(3, 150, 20, 150), block(8, 0, 1, 150)])
    assert _told_apart([block(0, 150, 8, 150), block(1, 0, 7, 150)])      # the later one is further left
    assert _told_apart([block(0, 0, 1, 100), block(0, 100, 8, 100)])      # one row of it
    assert _told_apart([block(0, 50, 8, 200), block(0, 250, 8, 100)])     # into the next row's first columns
    assert _told_apart([block(0, 100, 1, 250), block(0, 50, 8, 1)])
    # into blocks of the same matrix, and of another
    assert _told_apart([block(0, 0, 8, 100), block(0, 100, 8, 50)], [block(0, 150, 8, 100), block(0, 250, 8, 50)])
    assert _told_apart([block(0, 0, 8, 100)] * 2, [_slice(0, c, 8, 100, 777, dt, B) for c in (5, 105)])


@pytest.mark.parametrize("dt", [0, 1])
def test_clip_finds_blocks_that_meet(dt):
    def block(*a):
        return _slice(*a, 300, dt)
    for bad in ([block(0, 0, 8, 100), block(0, 99, 8, 100)], [block(0, 0, 8, 101), block(7, 100, 8, 100)],
                [block(0, 50, 8, 200), block(0, 250, 8, 101)],             # past the row's end
                [block(0, 0, 8, 100), block(0, 100, 8, 100), block(5, 199, 1, 1)],
                [block(0, 100, 1, 251), block(0, 50, 8, 1)],
                [block(0, 0, 8, 100), _slice(0, 150, 8, 100, 299, dt)],   # other strides: their extents
                [block(0, 0, 8, 100), (_slice(0, 150, 1, 1, 1, dt)[0], 1, 301, 301, dt)]):
        assert not _told_apart(bad) and not _told_apart(bad[::-1])
    assert not _told_apart([block(0, 0, 8, 100)], [block(0, 99, 8, 100)])
    # one pair of many blocks
    many = [block(0, 3 * i, 500, 3) for i in range(100)]
    assert _told_apart(many)
    assert not _told_apart(many + [block(499, 150, 1, 1)]) and _told_apart(many + [block(500, 150, 1, 1)])


def test_clip_blocks_against_sets_of_elements():
    """Random pairs of blocks, the check against the sets of their elements."""
    import random
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(2000):
        ld = rng.randint(1, 9)
        pair, sets = [], []
        for _ in range(2):
            at, rows, cols = rng.randint(0, 40), rng.randint(2, 5), rng.randint(1, ld)
            pair.append(_slice(0, at, rows, cols, ld, 1))
            sets.append({at + i * ld + j for i in range(rows) for j in range(cols)})
            if cols == ld:
                pair.pop()  # no gaps: a single row of all
                pair.append(_slice(0, at, 1, rows * cols, rows * cols, 1))
        meet = bool(sets[0] & sets[1])
        extents = max(map(min, sets)) <= min(map(max, sets))
        exact = all(p[1] > 1 for p in pair)
        assert _told_apart(pair) == (not (meet if exact else extents)), (ld, pair)
        seen[meet] += exact
    assert min(seen) > 100
