"""Every way a product of the linear layers is cut (tile, whole or split, each
operation and type; test_host_linearcuts.py holds the sizes to it) against
float64 products on the GPU, elementwise within the derived bounds of
model_util."""
import math

import pytest
import torch

from linear_cuts import CUTS
from model_util import EVAL, OUT, SLOPE, U, gen, rand

pytestmark = pytest.mark.gpu


def layers():
    from paper_2609_38767_amd import layers as m
    return m


def _check(got, want, bound, what):
    assert got.shape == want.shape
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), float((got.double() - want).abs().max()))


def _product(a, b):
    """a @ b in float64 and the bound on its float32 form; b made contiguous."""
    a, b = a.double(), b.double().contiguous()
    return a @ b, 2 * (a.shape[1] + 8) * U * (a.abs() @ b.abs())


@pytest.mark.parametrize("cut", CUTS, ids=lambda c: "-".join(map(str, c)))
def test_cut(cut):
    op, dtype, n, i, o, _, _ = cut
    g = gen(CUTS.index(cut))
    if op == 0:
        x, w = rand(g, n, i, dtype=dtype), rand(g, o, i, dtype=dtype, std=i ** -0.5)
        b, r = rand(g, o, dtype=dtype), rand(g, n, o, dtype=dtype)
        y, z = layers().linear(x, w, b, act="gelu", residual=r, keep_preact=True)
        wz, e = _product(x, w.mT)
        wz = wz + b.double()
        e = e + 2 * U * wz.abs()
        _check(z, wz, e + OUT[dtype] * (wz.abs() + e), "z")
        want = wz * torch.special.ndtr(wz) + r.double()
        ey = SLOPE * e + EVAL * wz.abs()
        _check(y, want, ey + OUT[dtype] * (want.abs() + ey) + 2 * U * (want.abs() + r.double().abs()), "y")
        assert torch.equal(layers().linear(x, w, b, act="gelu", residual=r), y)
    elif op == 1:
        gr, w = rand(g, n, o, dtype=dtype), rand(g, o, i, dtype=dtype, std=o ** -0.5)
        z, r = rand(g, n, i, dtype=dtype, std=2.0), rand(g, n, i, dtype=dtype)
        d, p = layers().linear_input_grad(gr, w, residual=r, act="gelu", preact=z, both=True)
        wd, e = _product(gr, w)
        wd = wd + r.double()
        e = e + 2 * U * (wd.abs() + r.double().abs())
        _check(d, wd, e + OUT[dtype] * (wd.abs() + e), "d")
        v = z.double()
        want = wd * (torch.special.ndtr(v) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi))
        ep = SLOPE * e + EVAL * (wd.abs() + e) * (1 + v.abs())
        _check(p, want, ep + OUT[dtype] * (want.abs() + ep), "p")
        assert torch.equal(layers().linear_input_grad(gr, w, residual=r, act="gelu", preact=z), p)
    else:
        gr, x = rand(g, n, o, dtype=dtype), rand(g, n, i, dtype=dtype)
        dw, db = layers().linear_weight_grad(gr, x, bias=True)
        want, e = _product(gr.mT, x)
        _check(dw, want, e, "dw")
        G = gr.double()
        _check(db, G.sum(0), 2 * (n + 8) * U * G.abs().sum(0), "db")
        w0 = rand(g, o, i)
        acc = layers().linear_weight_grad(gr, x, out=w0.clone(), accumulate=True)
        want = want + w0.double()
        _check(acc, want, e + U * (want.abs() + e), "dw accumulated")
