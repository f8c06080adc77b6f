"""Pins of the oracle's token log probabilities, norm and clipping: closed forms,
finite differences and the e4m3 format's own table.  No GPU."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import clip, logprobs, rmsnorm

INF = np.inf


def test_uniform_and_two_way_rows():
    V = 10
    logp, H, stats, top, ids = logprobs.token_logprobs(np.full((1, V), 3.0), [4], 3)
    assert np.allclose(logp, -math.log(V)) and np.allclose(H, math.log(V))
    assert np.allclose(stats, [[3.0, math.log(V)]]) and ids.tolist() == [[0, 1, 2]]
    # p = (3/4, 1/4)
    Z = np.array([[math.log(3.0), 0.0, -INF]])
    logp, H, _, top, ids = logprobs.token_logprobs(Z, [2], 3)
    assert logp[0] == -INF and np.allclose(top[0, :2], np.log([0.75, 0.25])) and top[0, 2] == -INF
    assert np.allclose(H, -(0.75 * math.log(0.75) + 0.25 * math.log(0.25)))
    # twice the scale: odds 9 to 1
    assert np.allclose(np.exp(logprobs.log_p(Z, 2.0))[0], [0.9, 0.1, 0.0])


def test_shift_invariance_and_huge_logits():
    Z = np.random.default_rng(0).standard_normal((4, 50))
    assert np.allclose(logprobs.log_p(Z), logprobs.log_p(Z + 1000.0), atol=1e-10)
    low = np.full((1, 8), float(np.finfo(np.float32).min))
    assert np.allclose(logprobs.log_p(low), -math.log(8))


def test_special_rows():
    Z = np.zeros((4, 5))
    Z[0] = -INF
    Z[1, 2] = np.nan
    Z[2, 2] = INF
    logp, H, stats, top, ids = logprobs.token_logprobs(Z, [1, 1, 1, -1], 2)
    assert logp[0] == -INF and H[0] == 0 and (stats[0] == -INF).all() and ids[0].tolist() == [0, 1]
    for i in (1, 2):
        assert np.isnan([logp[i], H[i], *stats[i], *top[i]]).all() and (ids[i] == -1).all()
    assert logp[3] == 0.0 and np.isclose(H[3], math.log(5))
    d = logprobs.token_logprobs_backward(Z, [1, 1, 1, -1], g_logp=[1, 0, 1, 5])
    assert d[0].tolist() == [0, 1, 0, 0, 0] and (d[1] == 0).all() and np.isnan(d[2]).all()
    assert (d[3] == 0).all()


def test_ties_take_the_lower_id():
    Z = np.array([[1.0, 5.0, 5.0, -0.0, 0.0, 5.0]])
    assert logprobs.token_logprobs(Z, [0], 6)[4].tolist() == [[1, 2, 5, 0, 3, 4]]


@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_logit_gradient_against_differences(scale):
    r = np.random.default_rng(1)
    Z = r.standard_normal((3, 7))
    Z[1, 4] = -INF
    tok = np.array([2, 0, -1])
    gl, gh = r.standard_normal(3), r.standard_normal(3)

    def f(z):
        lp, H, *_ = logprobs.token_logprobs(z, tok, 0, scale)
        return float((gl * lp + gh * H).sum())

    d = logprobs.token_logprobs_backward(Z, tok, gl, gh, scale)
    assert np.allclose(d.sum(1), 0.0, atol=1e-14)  # the log probabilities ignore a shift
    for i, j in np.ndindex(Z.shape):
        if Z[i, j] == -INF:
            assert d[i, j] == 0
            continue
        a, b = Z.copy(), Z.copy()
        a[i, j] += 1e-5
        b[i, j] -= 1e-5
        assert abs((f(a) - f(b)) / 2e-5 - d[i, j]) < 1e-8
    w = r.random(3)
    lp, dz = logprobs.token_loss(Z, tok, w, scale)
    assert np.allclose(dz, logprobs.token_logprobs_backward(Z, tok, -w, None, scale))


def test_norm_closed_forms():
    Y, H = rmsnorm.rmsnorm(np.array([[3.0, -4.0]]), eps=0.0)
    assert np.allclose(Y, np.array([[3.0, -4.0]]) / math.sqrt(12.5)) and (H == [[3, -4]]).all()
    X = np.random.default_rng(2).standard_normal((4, 33))
    Y, _ = rmsnorm.rmsnorm(X, eps=0.0)
    assert np.allclose((Y * Y).mean(1), 1.0)
    assert np.allclose(rmsnorm.rmsnorm(5 * X, eps=0.0)[0], Y)
    Y2, H = rmsnorm.rmsnorm(X, w=np.full(33, 2.0), residual=X, eps=0.0)
    assert np.allclose(Y2, 2 * Y) and np.allclose(H, 2 * X)


def test_norm_gradient_against_differences():
    r = np.random.default_rng(3)
    H, dY, w, dH = r.standard_normal((2, 6)), r.standard_normal((2, 6)), r.standard_normal(6), \
        r.standard_normal((2, 6))

    def f(h, g):
        return float((rmsnorm.rmsnorm(h, g)[0] * dY).sum() + (h * dH).sum())

    dX, gw = rmsnorm.rmsnorm_backward(H, dY, w, dH)
    for i, j in np.ndindex(H.shape):
        e = np.zeros_like(H)
        e[i, j] = 1e-6
        assert abs((f(H + e, w) - f(H - e, w)) / 2e-6 - dX[i, j]) < 1e-8
    for j in range(6):
        e = np.zeros(6)
        e[j] = 1e-6
        assert abs((f(H, w + e) - f(H, w - e)) / 2e-6 - gw[j]) < 1e-8


def test_e4m3_table_and_rounding():
    """The oracle's table and its rounding against torch's type."""
    v = rmsnorm.e4m3_values()
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, t, equal_nan=True)
    x = np.concatenate([np.linspace(-448, 448, 20001), 2.0 ** np.linspace(-12, 8.8, 5000),
                        (v[:126] + v[1:127]) / 2])  # and every tie
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    x = x.astype(np.float32).astype(np.float64)
    assert np.array_equal(rmsnorm.round_e4m3(x), want)


def test_scales():
    Y = np.zeros((2, 300))
    Y[0, 5], Y[0, 130], Y[1, 299] = -4.48, 8.96, 448.0
    S = rmsnorm.scales(Y, 128)
    assert np.allclose(S, [[0.01, 0.02, 2.0 ** -100 / 448], [2.0 ** -100 / 448] * 2 + [1.0]])
    assert np.allclose(rmsnorm.scales(Y)[:, 0], [0.02, 1.0])
    assert rmsnorm.spread(S, 300, 128).shape == (2, 300)


def test_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    assert clip.sumsq(g) == 25.0
    norm, out = clip.clip(g, 25.0, 1.0)
    assert norm == 5.0 and np.allclose(out[0], [0.6, 0]) and np.allclose(out[1], 0.8)
    assert all((a == b).all() for a, b in zip(g, clip.clip(g, 25.0, 5.0)[1]))


def test_package_names():
    assert oracle.logprobs is logprobs and oracle.rmsnorm is rmsnorm and oracle.clip is clip
