"""Pins of the oracle's block norm, gated feed-forward block and orthogonalised updates: closed
forms, finite differences, singular values.  No GPU."""
import math

import numpy as np
import pytest

from oracle import blocknorm, gated_ff, orth, rmsnorm

RNG = np.random.default_rng


def _difference(f, x, direction, h=1e-6):
    return (f(x + h * direction) - f(x - h * direction)) / (2 * h)


def test_block_norm_is_the_norm_without_post_and_gate():
    r = RNG(0)
    X, R, w = r.standard_normal((3, 7)), r.standard_normal((3, 7)), r.standard_normal(7)
    Y, H = blocknorm.block_norm(X, R, w, post=False)
    y, h = rmsnorm.rmsnorm(X, w, R)
    assert np.allclose(Y, y) and np.allclose(H, h)


def test_block_norm_of_equal_values():
    # a row of twos has root mean square 2: z = 1, gate sigmoid(0) = 1/2, h = 3 + 1/2
    X, R = np.full((1, 4), 2.0), np.full((1, 4), 6.0)
    Y, H = blocknorm.block_norm(X, R, gate=np.zeros(4), fn="sigmoid", alpha=0.5, eps=0.0)
    assert np.allclose(H, 3.5) and np.allclose(Y, 1.0)


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate,fn", [(None, "none"), ("row", "none"), ("row", "sigmoid"), ("token", "sigmoid")])
def test_block_norm_gradients_against_differences(post, gate, fn):
    r = RNG(1)
    n, d, alpha = 4, 6, 0.7
    X, R, dY, dH = (r.standard_normal((n, d)) for _ in range(4))
    w, w1 = r.standard_normal(d), r.standard_normal(d)
    g = None if gate is None else r.standard_normal(d if gate == "row" else (n, d))

    def loss(X=X, R=R, w=w, w1=w1, g=g):
        Y, H = blocknorm.block_norm(X, R, w, w1, post, g, fn, alpha)
        return (Y * dY).sum() + (H * dH).sum()

    H = blocknorm.block_norm(X, R, w, w1, post, g, fn, alpha)[1]
    b = blocknorm.block_norm_backward(X, H, dY, w, w1, post, g, fn, alpha, dH)
    for key, name, at, grad in (("X", "X", X, b["dX"]), ("R", "R", R, b["dR"]), ("w", "w", w, b["gw"]),
                                ("w1", "w_post", w1, b["gw_post"]), ("g", "gate", g, b["dgate"])):
        if at is None or (key == "w1" and not post):
            continue
        v = r.standard_normal(at.shape)
        grad = grad.sum(0) if key == "g" and gate == "row" else grad
        assert math.isclose((grad * v).sum(), _difference(lambda t: loss(**{key: t}), at, v),
                            rel_tol=1e-6, abs_tol=1e-7), name


def test_activations():
    a, s = gated_ff.act("silu", [0.0, math.log(3.0), -800.0])
    assert np.allclose(a, [0.0, 0.75 * math.log(3.0), 0.0]) and s[0] == 0.5 and s[2] == 0
    a, s = gated_ff.act("gelu", [0.0, 1.0, -1.0])
    assert np.allclose(a, [0.0, 0.8413447460685429, -0.15865525393145707]) and s[0] == 0.5
    a, s = gated_ff.act("relu", [-1.0, 0.0, 2.0])
    assert a.tolist() == [0, 0, 2] and s.tolist() == [0, 0, 1]


@pytest.mark.parametrize("name", ["silu", "gelu", "relu"])
def test_gated_ff_gradients_against_differences(name):
    r = RNG(2)
    X, Wg, Wu, dH = (r.standard_normal(s) for s in ((3, 5), (5, 4), (5, 4), (3, 4)))
    _, G, U = gated_ff.gated_ff(X, Wg, Wu, name)
    dG, dU = gated_ff.projections_backward(G, U, dH, name)
    dX, gWg, gWu = gated_ff.products_backward(X, Wg, Wu, dG, dU)
    for k, (at, grad) in enumerate(((X, dX), (Wg, gWg), (Wu, gWu))):
        v = r.standard_normal(at.shape)

        def loss(t):
            args = [X, Wg, Wu]
            args[k] = t
            return (gated_ff.gated_ff(*args, name)[0] * dH).sum()
        assert math.isclose((grad * v).sum(), _difference(loss, at, v), rel_tol=1e-6, abs_tol=1e-7)


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (6, 6), (1, 7), (7, 1), (1, 1)])
def test_orthogonalize_acts_on_singular_values(shape):
    M = RNG(3).standard_normal(shape)
    assert np.allclose(orth.orthogonalize(M), orth.by_singular_values(M), atol=1e-10)


def test_five_steps_take_singular_values_towards_one():
    s = orth.f(np.linspace(1 / 300, 1.0, 4000), 5)
    assert 0.68 < s.min() and s.max() < 1.21
    assert np.allclose(orth.orthogonalize(np.zeros((3, 4))), 0.0)


def test_the_update_keeps_the_column_space():
    r = RNG(4)
    U = np.linalg.qr(r.standard_normal((20, 4)))[0]
    G, M = U @ r.standard_normal((4, 30)), U @ r.standard_normal((4, 30))
    W0 = U @ r.standard_normal((4, 30))
    W, m = orth.muon_step(W0, G, M, 0.1, decay=0.01)
    assert np.allclose(U @ (U.T @ W), W) and np.allclose(m, 0.95 * M + G)
    assert not np.allclose(W, W0)


def test_muon_without_nesterov():
    r = RNG(5)
    G, M = r.standard_normal((4, 6)), r.standard_normal((4, 6))
    m, b = orth.momentum(M, G, 0.5, False)
    assert np.allclose(b, 0.5 * M + G) and np.allclose(m, b)
    assert np.allclose(orth.momentum(M, G, 0.5)[1], G + 0.5 * m)
