"""Root-mean-square norm and its gradient, 8-bit rows and weights, the products
of 8-bit operands and the linear layers of experts in float64 (oracle side).

With h = x + r and u = (mean h^2 + eps)^(-1/2): y = h u w.  From g = dL/dy,
dL/dh_k = u w_k g_k - h_k u^3 / d sum_j g_j w_j h_j  (du/dh_k = -u^3 h_k / d), and
dL/dw = sum over rows of g h u.
"""
import numpy as np

from . import model as om

BLOCK, MOST, LEAST = 128, 448.0, 2.0 ** -126


def rms_norm(x, w, r=None, eps=1e-6):
    """(y, h, u) of rows x [n, d]."""
    h = np.asarray(x, np.float64)
    if r is not None:
        h = h + np.asarray(r, np.float64)
    u = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    return h * u * np.asarray(w, np.float64), h, u


def rms_norm_grad(g, h, w, p=None, eps=1e-6):
    """(gradient of h, gradient of w)."""
    g, h, w = (np.asarray(v, np.float64) for v in (g, h, w))
    u = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    d = u * (g * w - h * u * u * (g * w * h).mean(-1, keepdims=True))
    if p is not None:
        d = d + np.asarray(p, np.float64)
    return d, (g * h * u).sum(0)


def e4m3(v):
    """The e4m3 value nearest to v, ties to even: 3 bits behind the leading one,
    steps of 2^-9 below 2^-6, magnitudes over 448 + 16 become NaN."""
    v = np.asarray(v, np.float64)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -30))), -6.0) - 3.0)
    q = np.round(v / step) * step  # numpy rounds halves to even
    return np.where(np.abs(q) > MOST, np.nan, q)


def scales(v, rows):
    """float32 scales of v [n, d] by groups of `rows` x 128."""
    n, d = v.shape
    top = np.maximum.reduceat(np.abs(np.asarray(v, np.float32)), np.arange(0, d, BLOCK), axis=1)
    top = np.maximum.reduceat(top, np.arange(0, n, rows), axis=0) if rows > 1 else top
    return np.maximum(top / np.float32(MOST), np.float32(LEAST))


def spread(s, n, d, rows):
    """Scales of every element [n, d]."""
    return np.repeat(np.repeat(s, rows, 0)[:n], BLOCK, 1)[:, :d]


def quantize(v, rows=1):
    """(values, scales) of float32 v [n, d]; the division is float32's."""
    v = np.asarray(v, np.float32)
    s = scales(v, rows)
    return e4m3(v / spread(s, *v.shape, rows)), s


def expert_rows(offsets, n):
    """[(expert or None, slice)] of all rows."""
    o = [int(v) for v in offsets]
    own = [(e, slice(a, b)) for e, (a, b) in enumerate(zip(o, o[1:]))]
    return [(None, slice(0, o[0]))] + own + [(None, slice(o[-1], n))]


def expert_linear(x, w, offsets, b=None, kind="none", r=None):
    """(y, z) of rows sorted by expert."""
    x = np.asarray(x, np.float64)
    z = np.zeros((len(x), w.shape[1]))
    for e, at in expert_rows(offsets, len(x)):
        if e is not None:
            z[at] = om.linear(x[at], w[e], None if b is None else b[e])[1]
    y = om.act(z, kind)
    return (y if r is None else y + np.asarray(r, np.float64)), z


def expert_input_grad(g, w, offsets, r=None, kind="none", z=None):
    """(d, p): the gradient of the rows and that times the slope at z."""
    g = np.asarray(g, np.float64)
    d = np.zeros((len(g), w.shape[2]))
    for e, at in expert_rows(offsets, len(g)):
        if e is not None:
            d[at] = g[at] @ np.asarray(w[e], np.float64)
    if r is not None:
        d = d + np.asarray(r, np.float64)
    return d, (d if kind == "none" else d * om.act_slope(z, kind))


def expert_weight_grad(g, x, offsets):
    """(dw [experts, d_out, d_in], db [experts, d_out])."""
    at = [s for e, s in expert_rows(offsets, len(g)) if e is not None]
    g, x = np.asarray(g, np.float64), np.asarray(x, np.float64)
    return np.stack([g[s].T @ x[s] for s in at]), np.stack([g[s].sum(0) for s in at])
