"""The model-side operators in float64 (oracle side): embedding lookup and its
table gradient, linear layers with bias, activation and residual and their
backward products, the gradient norm and clipping.

A linear layer is z = W x + b per row, y = act(z) + r; with g = dL/dz the chain
rule gives dL/dx = g W, dL/dW = sum over rows of g x^T (Eq. (1) summed over the
batch) and dL/db = sum of g.
"""
import math

import numpy as np

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _erf(x):
    return np.vectorize(math.erf, otypes=[np.float64])(x)


def _logistic(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def act(z, kind):
    z = np.asarray(z, dtype=np.float64)
    if kind == "relu":
        return np.where(z < 0, 0.0, z)
    if kind == "gelu":
        return z * 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if kind == "silu":
        return z * _logistic(z)
    assert kind == "none"
    return z


def act_slope(z, kind):
    z = np.asarray(z, dtype=np.float64)
    if kind == "relu":
        return np.where(z <= 0, 0.0, 1.0)
    if kind == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if kind == "silu":
        s = _logistic(z)
        return s * (1.0 + z * (1.0 - s))
    assert kind == "none"
    return np.ones_like(z)


def linear(x, w, b=None, kind="none", r=None):
    """(y, z) of rows x [n, d_in] and weight w [d_out, d_in]."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if b is not None:
        z = z + np.asarray(b, np.float64)
    y = act(z, kind)
    return (y if r is None else y + np.asarray(r, np.float64)), z


def linear_input_grad(g, w, r=None, kind="none", z=None):
    """(d, p): d = g W + r and p = d * act'(z)."""
    d = np.asarray(g, np.float64) @ np.asarray(w, np.float64)
    if r is not None:
        d = d + np.asarray(r, np.float64)
    if kind == "none":
        return d, d
    return d, d * act_slope(z, kind)


def linear_weight_grad(g, x):
    """(dW, db)."""
    g, x = np.asarray(g, np.float64), np.asarray(x, np.float64)
    return g.T @ x, g.sum(0)


def embedding(table, tokens, scale=1.0):
    table = np.asarray(table, np.float64)
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[i] = scale * table[t]
    return out


def embedding_grad(grad_out, tokens, vocab, scale=1.0):
    grad_out = np.asarray(grad_out, np.float64)
    out = np.zeros((vocab, grad_out.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < vocab:
            out[t] += scale * grad_out[i]
    return out


def clip(grads, max_norm):
    """(scaled gradients, norm, coefficient)."""
    norm = math.sqrt(sum(float(np.square(np.asarray(g, np.float64)).sum()) for g in grads))
    coef = 1.0 if max_norm == math.inf else min(1.0, max_norm / (norm + 1e-6))
    return [np.asarray(g, np.float64) * coef for g in grads], norm, coef
