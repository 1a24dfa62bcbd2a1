"""The float64 model-side operators: gradients against differences of the
forward pass, and hand-computed values."""
import math

import numpy as np
import pytest

from oracle import model as om


def _central(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


# a central difference with h = 1e-6 is off by h^2 f'''/6 ~ 1e-12 and by
# rounding 2^-53 |f| / h ~ 1e-9 for |f| of a few tens
TOL = 1e-7


@pytest.mark.parametrize("kind", om.ACTS)
def test_activation_slopes(kind):
    z = np.array([-6.0, -2.5, -0.7, -1e-3, 1e-3, 0.3, 1.9, 5.0])
    d = (om.act(z + 1e-6, kind) - om.act(z - 1e-6, kind)) / 2e-6
    assert np.abs(om.act_slope(z, kind) - d).max() < TOL


def test_activation_values():
    assert om.act(np.array([0.0, -3.0, 2.0]), "relu").tolist() == [0.0, 0.0, 2.0]
    assert om.act(1.0, "gelu") == pytest.approx(0.8413447460685429, abs=1e-15)  # Phi(1)
    assert om.act(1.0, "silu") == pytest.approx(1 / (1 + math.exp(-1)), abs=1e-15)
    assert om.act(1.0, "gelu_tanh") == pytest.approx(0.841192, abs=1e-6)
    assert om.act_slope(0.0, "gelu") == 0.5 and om.act_slope(0.0, "silu") == 0.5


@pytest.mark.parametrize("kind", om.ACTS)
def test_linear_gradients_by_differences(kind):
    """Two layers with a residual around the second: every gradient of a fixed
    linear functional of the output."""
    rng = np.random.default_rng(3)
    n, d, h = 3, 4, 5
    x, w1, b1, w2 = rng.normal(size=(n, d)), rng.normal(size=(h, d)), rng.normal(size=h), rng.normal(size=(d, h))
    c = rng.normal(size=(n, d))  # dL/dy

    def loss(x, w1, b1, w2):
        h1, _ = om.linear(x, w1, b1, kind)
        y, _ = om.linear(h1, w2, None, "none", x)
        return float((c * y).sum())

    h1, z1 = om.linear(x, w1, b1, kind)
    _, g1 = om.linear_input_grad(c, w2, None, kind, z1)
    dx, _ = om.linear_input_grad(g1, w1, c)  # the residual path brings c itself
    dw1, db1 = om.linear_weight_grad(g1, x)
    dw2, _ = om.linear_weight_grad(c, h1)
    for got, f, at in ((dx, lambda v: loss(v, w1, b1, w2), x), (dw1, lambda v: loss(x, v, b1, w2), w1),
                       (db1, lambda v: loss(x, w1, v, w2), b1), (dw2, lambda v: loss(x, w1, b1, v), w2)):
        assert np.abs(got - _central(f, at)).max() < TOL


def test_embedding_gradient_by_differences():
    rng = np.random.default_rng(4)
    table, tokens = rng.normal(size=(6, 3)), np.array([4, 0, 4, -1, 6, 2, 4])
    c = rng.normal(size=(7, 3))
    got = om.embedding_grad(c, tokens, 6, 2.5)
    want = _central(lambda t: float((c * om.embedding(t, tokens, 2.5)).sum()), table)
    assert np.abs(got - want).max() < TOL
    assert not got[[1, 3, 5]].any()


def test_clip():
    g = [np.array([3.0]), np.array([[0.0, 4.0]]), np.zeros(0)]
    out, norm, coef = om.clip(g, 1.0)
    assert norm == 5.0 and coef == pytest.approx(1 / (5 + 1e-6))
    assert math.sqrt(sum(float((o ** 2).sum()) for o in out)) == pytest.approx(1.0, rel=1e-6)
    assert om.clip(g, 7.0)[2] == 1.0 and om.clip(g, math.inf)[2] == 1.0
