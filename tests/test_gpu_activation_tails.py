"""Activations and their slopes relative to their own size, where they decay.

The reference forms Phi by erfc and the logistic function by exp(-|x|), so it
keeps its digits in the tails.  Relative bounds, U the unit roundoff of float32
and x the argument of the logistic function or of exp:

* gelu, float32: erfc's argument is off by 2 U of itself, erfc by (z^2 + 1)
  times that, and 32 U cover the library's erfc and the products around it; the
  density exp(-z^2 / 2) by z^2 U and its own 32 U.
* gelu, bf16 results: the fit of Phi is within 2^-16 of it (exp of a rounded
  argument included); 2^-15 with the products around it.
* silu and the tanh form: x has 6 U (a sum of two terms of one sign and the
  products in them; three products more where exp is formed by exp2), exp |x|
  times that, 32 U for the rest; silu's x is z itself.

A slope is a sum of two terms and its error that of both.  exp below 2^-126 may
read as zero: |z| 2^-126 of a value, times 2 (1 + z^2) for the derivative of
the tanh form's argument."""
import math

import numpy as np
import pytest
import torch

from model_util import DT, OUT, U, check, host

pytestmark = pytest.mark.gpu


def layers():
    from paper_2609_38767_amd import layers as m
    return m


def _logistic(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def reference(z, kind, dtype):
    """value, slope, and the bounds on their errors before the results are rounded."""
    least = 2.0 ** -126
    if kind == "gelu":
        phi = 0.5 * np.array([math.erfc(-v / math.sqrt(2.0)) for v in z])
        density = z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
        rel = (2 * (z * z + 1) + 32) * U if dtype == "f32" else 2.0 ** -15
        return z * phi, phi + density, rel * np.abs(z * phi) + np.abs(z) * least, \
            rel * (phi + np.abs(density)) + (1 + np.abs(z)) * least
    c, k = math.sqrt(2.0 / math.pi), 0.044715
    x, dx = (z, np.ones_like(z)) if kind == "silu" else (2 * c * (z + k * z ** 3), 2 * c * (1 + 3 * k * z * z))
    s, t = _logistic(x), _logistic(-x)
    rel = ((6 if dtype == "f32" else 9) * np.abs(x) + 32) * U
    return z * s, s + z * dx * s * t, rel * z * s * np.sign(z) + np.abs(z) * least, \
        2 * rel * (s + np.abs(z * dx) * s * t) + (1 + np.abs(z) * 2 * (1 + z * z)) * least


def _points(dtype):
    """Every bfloat16 from 2^-8 to 40 in magnitude, or as many float32 values; zeros and the smallest magnitudes."""
    bits = np.arange(int(np.float32(2.0 ** -8).view(np.uint32)) >> 16, (int(np.float32(40.0).view(np.uint32)) >> 16) + 1)
    v = (bits.astype(np.uint32) << 16).view(np.float32)
    if dtype == "f32":
        v = np.concatenate([v, np.linspace(2.0 ** -8, 40.0, 4001, dtype=np.float32)])
    v = np.concatenate([v, np.float32([0.0, 1e-6, 1e-30])])
    return torch.from_numpy(np.concatenate([v, -v])).to(DT[dtype]).cuda()[:, None].contiguous()


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tails(kind, dtype):
    z = _points(dtype)
    one = torch.ones(1, 1, dtype=DT[dtype], device="cuda")
    with np.errstate(under="ignore"):
        value, slope, ev, es = (a[:, None] for a in reference(host(z)[:, 0], kind, dtype))
    check(layers().linear(z, one, act=kind), value, ev + OUT[dtype] * (np.abs(value) + ev) + 2.0 ** -134, "value")
    p = layers().linear_input_grad(torch.ones_like(z), one, act=kind, preact=z)
    check(p, slope, es + OUT[dtype] * (np.abs(slope) + es) + 2.0 ** -134, "slope")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_wide_and_few_row_forms_share_the_tails(dtype):
    """The same values through the few-row form and through tiles: an identity weight carries z to every column."""
    z = _points(dtype)[:, 0]
    n = z.numel()
    eye = torch.eye(max(n, 2048), dtype=DT[dtype], device="cuda")[:, :n].contiguous()
    want = layers().linear(z[:, None].contiguous(), torch.ones(1, 1, dtype=DT[dtype], device="cuda"), act="gelu")[:, 0]
    for rows in (1, 4, 64, 200):
        y = layers().linear(z.expand(rows, n).contiguous(), eye, act="gelu")
        assert torch.equal(y[:, :n], want.expand(rows, n))
