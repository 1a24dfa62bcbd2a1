"""The oracle of the norm, of 8-bit values and of the experts' layers against
differences, published values of the format and plain loops."""
import numpy as np
import pytest
import torch

from oracle import block as ob
from oracle import model as om


@pytest.mark.parametrize("n,d", [(1, 1), (3, 2), (4, 7), (2, 33)])
def test_norm_gradients_are_differences(n, d):
    rng = np.random.default_rng(n * 100 + d)
    x, r, g, p = (rng.standard_normal((n, d)) for _ in range(4))
    w, eps = 1 + 0.3 * rng.standard_normal(d), 0.05

    def loss(x, w):
        y, h, _ = ob.rms_norm(x, w, r, eps)
        return (y * g).sum() + (h * p).sum()
    _, h, _ = ob.rms_norm(x, w, r, eps)
    dx, dw = ob.rms_norm_grad(g, h, w, p, eps)
    # central differences of step 1e-5: off by step^2 times a third derivative, which powers of u <= eps^-1/2 = 4.5
    # bound by 1e4 |g w| here, and by 2^-52 |loss| / step
    tol = 1e-10 * 1e4 * (np.abs(g).max() * np.abs(w).max() + 1) * d + 2 ** -50 * 100 / 1e-5
    for i in range(n):
        for j in range(d):
            e = np.zeros((n, d))
            e[i, j] = 1e-5
            assert abs((loss(x + e, w) - loss(x - e, w)) / 2e-5 - dx[i, j]) < tol
    for j in range(d):
        e = np.zeros(d)
        e[j] = 1e-5
        assert abs((loss(x, w + e) - loss(x, w - e)) / 2e-5 - dw[j]) < tol


def test_e4m3_is_the_format():
    """Every value stands for itself, the middle of two neighbours goes to the even one, all else to the nearer."""
    codes = torch.arange(127, dtype=torch.uint8)
    v = codes.view(torch.float8_e4m3fn).double().numpy()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[-1] == 448
    assert np.array_equal(ob.e4m3(v), v) and np.array_equal(ob.e4m3(-v), -v)
    mid = (v[:-1] + v[1:]) / 2
    assert np.array_equal(ob.e4m3(mid), np.where(np.arange(126) % 2 == 0, v[:-1], v[1:]))
    assert np.array_equal(ob.e4m3(mid * (1 + 1e-9)), v[1:]) and np.array_equal(ob.e4m3(mid * (1 - 1e-9)), v[:-1])
    assert ob.e4m3(463.9) == 448 and np.isnan(ob.e4m3(470.0))


def test_quantize_groups():
    rng = np.random.default_rng(3)
    v = rng.standard_normal((130, 300)).astype(np.float32)
    v[:, :128][5] = 0
    q, s = ob.quantize(v)
    assert s.shape == (130, 3) and s[5, 0] == np.float32(2.0 ** -126) and not q[5, :128].any()
    assert s[7, 2] == np.abs(v[7, 256:]).max() / np.float32(448)
    q, s = ob.quantize(v, 128)
    assert s.shape == (2, 3) and s[1, 1] == np.abs(v[128:, 128:256]).max() / np.float32(448)
    err = np.abs(q * ob.spread(s, 130, 300, 128) - v)
    assert (err <= np.maximum(2.0 ** -4 * np.abs(v), 2.0 ** -10 * s.max()) * (1 + 1e-6)).all()


@pytest.mark.parametrize("offsets", [(0, 3, 3, 8), (2, 2, 5, 6), (0, 0, 0, 0), (8, 8, 8, 8)])
def test_experts_row_by_row(offsets):
    rng = np.random.default_rng(1)
    x, w, b, r = (rng.standard_normal(s) for s in ((8, 4), (3, 5, 4), (3, 5), (8, 5)))
    y, z = ob.expert_linear(x, w, offsets, b, "silu", r)
    g = rng.standard_normal((8, 5))
    d, _ = ob.expert_input_grad(g, w, offsets)
    dw, db = ob.expert_weight_grad(g, x, offsets)
    ww, wb = np.zeros_like(w), np.zeros_like(b)
    for t in range(8):
        e = [k for k in range(3) if offsets[k] <= t < offsets[k + 1]]
        zt = w[e[0]] @ x[t] + b[e[0]] if e else np.zeros(5)
        assert np.allclose(z[t], zt, atol=1e-14) and np.allclose(y[t], om.act(zt, "silu") + r[t], atol=1e-14)
        assert np.allclose(d[t], w[e[0]].T @ g[t] if e else 0, atol=1e-14)
        if e:
            ww[e[0]] += np.outer(g[t], x[t])
            wb[e[0]] += g[t]
    assert np.allclose(dw, ww, atol=1e-13) and np.allclose(db, wb, atol=1e-13)
