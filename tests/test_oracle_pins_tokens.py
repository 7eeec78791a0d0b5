"""Pins of oracle/tokens_oracle.py: closed forms, dense one-hot products, central differences of every gradient (CPU)."""
import numpy as np

import oracle


def _diff(f, x, h=1e-6):
    """Central differences of the scalar f at x."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_embedding_is_the_one_hot_product_and_its_gradient_the_transposed_one():
    rng = np.random.default_rng(1)
    table, ids, dy = rng.normal(size=(7, 5)), np.array([3, 0, 3, -1, 7, 6, 3]), rng.normal(size=(7, 5))
    onehot = np.array([[float(i == v) for v in range(7)] for i in ids])
    np.testing.assert_allclose(oracle.embedding(table, ids, 2.5), 2.5 * onehot @ table, rtol=1e-15)
    np.testing.assert_allclose(oracle.embedding_bwd(dy, ids, 7, 2.5), 2.5 * onehot.T @ dy, rtol=1e-14)
    assert (oracle.embedding(table, ids)[[3, 4]] == 0).all()
    np.testing.assert_allclose(_diff(lambda t: float((oracle.embedding(t, ids, 2.5) * dy).sum()), table), oracle.embedding_bwd(dy, ids, 7, 2.5),
                               atol=1e-8)


def test_layer_norm_closed_forms():
    y, mean, rstd = oracle.layer_norm(np.array([[1.0, 3.0]]), eps=0.0)
    np.testing.assert_allclose(y, [[-1.0, 1.0]])
    np.testing.assert_allclose((mean[0], rstd[0]), (2.0, 1.0))
    y, mean, rstd = oracle.layer_norm(np.full((2, 9), 4.0), np.full(9, 7.0), np.arange(9.0), eps=0.25)
    np.testing.assert_allclose(y, np.tile(np.arange(9.0), (2, 1)))        # a constant row: beta
    np.testing.assert_allclose(rstd, 2.0)
    rng = np.random.default_rng(2)
    y, _, _ = oracle.layer_norm(rng.normal(size=(4, 300)) * 9 + 100, eps=0.0)
    np.testing.assert_allclose(y.mean(1), 0, atol=1e-12)
    np.testing.assert_allclose((y ** 2).mean(1), 1, rtol=1e-12)


def test_layer_norm_bwd_matches_central_differences():
    rng = np.random.default_rng(3)
    x, gamma, beta, dy = rng.normal(size=(3, 6)), rng.normal(size=6), rng.normal(size=6), rng.normal(size=(3, 6))
    _, mean, rstd = oracle.layer_norm(x, gamma, beta, 0.1)
    dx, dgamma, dbeta = oracle.layer_norm_bwd(x, gamma, mean, rstd, dy)
    loss = lambda a, g, b: float((oracle.layer_norm(a, g, b, 0.1)[0] * dy).sum())
    np.testing.assert_allclose(dx, _diff(lambda a: loss(a, gamma, beta), x), atol=1e-8)
    np.testing.assert_allclose(dgamma, _diff(lambda a: loss(x, a, beta), gamma), atol=1e-8)
    np.testing.assert_allclose(dbeta, _diff(lambda a: loss(x, gamma, a), beta), atol=1e-8)
    np.testing.assert_allclose(oracle.layer_norm_bwd(x, None, mean, rstd, dy)[0], oracle.layer_norm_bwd(x, np.ones(6), mean, rstd, dy)[0])


def test_linear_xent_closed_forms():
    loss, lse = oracle.linear_xent(np.zeros((3, 4)), np.ones((10, 4)), [0, 9, -1])
    np.testing.assert_allclose(lse, np.log(10.0))
    np.testing.assert_allclose(loss, [np.log(10.0), np.log(10.0), 0.0])
    loss, lse = oracle.linear_xent([[800.0]], [[1.0], [0.0]], [1])              # no overflow
    np.testing.assert_allclose((loss[0], lse[0]), (800.0, 800.0))
    x, w = np.random.default_rng(4).normal(size=(5, 3)), np.random.default_rng(5).normal(size=(8, 3))
    p = oracle.softmax(x @ w.T)
    np.testing.assert_allclose(oracle.linear_xent(x, w, [0, 1, 2, 3, 7])[0], -np.log(p[np.arange(5), [0, 1, 2, 3, 7]]), rtol=1e-12)


def test_linear_xent_bwd_matches_central_differences():
    rng = np.random.default_rng(6)
    x, w, dloss = rng.normal(size=(4, 3)), rng.normal(size=(6, 3)), np.array([0.5, -2.0, 3.0, 1.0])
    labels = np.array([2, 5, -100, 2])
    _, lse = oracle.linear_xent(x, w, labels)
    dx, dw = oracle.linear_xent_bwd(x, w, labels, lse, dloss)
    loss = lambda a, b: float((oracle.linear_xent(a, b, labels)[0] * dloss).sum())
    np.testing.assert_allclose(dx, _diff(lambda a: loss(a, w), x), atol=1e-8)
    np.testing.assert_allclose(dw, _diff(lambda a: loss(x, a), w), atol=1e-8)
    assert (dx[2] == 0).all()
