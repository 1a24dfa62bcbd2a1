"""Linear layers at sizes that take the 256 x 256 tiles, several rounds of the
buffers and ragged edges, and the few-row form, against float64 products on the
GPU, elementwise within the same derived bounds as the small sizes."""
import numpy as np
import pytest
import torch

from model_util import DT, EVAL, OUT, SLOPE, U, check, gen, host, product_bound, rand
from oracle import model as om

pytestmark = pytest.mark.gpu


def layers():
    from paper_2609_38767_amd import layers as m
    return m


def _check(got, want, bound):
    assert got.shape == want.shape
    bad = ~((got.double() - want).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float((got.double() - want).abs().max()))


def _bound(a, b):
    """2 (K + 8) U |a| |b| as in model_util, for float64 tensors."""
    return 2 * (a.shape[1] + 8) * U * (a.abs() @ b.abs())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cut", ["whole", "ragged", "odd"])
def test_large_tiles(cut, dtype):
    big, deep = {"whole": (4096, 1536), "ragged": (4088, 1480), "odd": (4085, 1483)}[cut]
    g = gen(61)
    x, w, b = rand(g, big, deep, dtype=dtype), rand(g, big, deep, dtype=dtype), rand(g, big, dtype=dtype)
    y = layers().linear(x, w, b)
    X, W = x.double(), w.double()
    want = X @ W.mT.contiguous() + b.double()
    e = _bound(X, W.mT.contiguous()) + 2 * U * want.abs()
    _check(y, want, e + OUT[dtype] * (want.abs() + e))
    wt = rand(g, deep, big, dtype=dtype)
    d = layers().linear_input_grad(x, wt)
    want = X @ wt.double()
    e = _bound(X, wt.double()) + 2 * U * want.abs()
    _check(d, want, e + OUT[dtype] * (want.abs() + e))
    gt, xt = rand(g, deep, big, dtype=dtype), rand(g, deep, big, dtype=dtype)
    dw, db = layers().linear_weight_grad(gt, xt, bias=True)
    G = gt.double().mT.contiguous()
    _check(dw, G @ xt.double(), _bound(G, xt.double()))
    _check(db, G.sum(1), 2 * (deep + 8) * U * G.abs().sum(1))
    assert torch.equal(layers().linear_weight_grad(gt, xt), dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("size,pad,offset", [((4096, 2048), 0, 0), ((8, 2050), 0, 0), ((777, 3001), 0, 0),
                                             ((2056, 2052), 8, 8), ((1000, 2051), 3, 1), ((1, 4099), 0, 0)])
def test_few_rows(rows, size, pad, offset, dtype):
    """Rows against a wide layer: every number of rows that has a form of its own, aligned and not."""
    i, o = size
    g = gen(67 + rows)
    x, w = rand(g, rows, i, dtype=dtype, pad=pad, offset=offset), rand(g, o, i, dtype=dtype, pad=pad, offset=offset)
    b, r = rand(g, o, dtype=dtype), rand(g, rows, o, dtype=dtype, pad=pad)
    y, z = layers().linear(x, w, b, act="silu", residual=r, keep_preact=True)
    want, wz = om.linear(host(x), host(w), host(b), "silu", host(r))
    e = product_bound(host(x), host(w).T) + 2 * U * np.abs(wz)
    check(z, wz, e + OUT[dtype] * (np.abs(wz) + e))
    ey = SLOPE * e + EVAL * np.abs(wz)
    check(y, want, ey + OUT[dtype] * (np.abs(want) + ey) + 2 * U * (np.abs(want) + np.abs(host(r))))
    assert torch.equal(layers().linear(x, w, b, act="silu", residual=r), y)
    bad = w.clone()
    bad[o - 1, 0] = float("nan")  # the last row's own output only
    y = layers().linear(x, bad, b)
    assert torch.isnan(y[:, o - 1]).all() and torch.isfinite(y[:, : o - 1]).all()


def test_rows_past_32_bit_offsets():
    """A factor block of more than 4 GiB: the last rows of G and X take part in the weight gradient, and its
    rows get their outputs."""
    n, i, o = 70_000, 72, 32_768  # G: 4.6 GB of bfloat16
    g = torch.zeros(n, o, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(n, i, dtype=torch.bfloat16, device="cuda")
    g[n - 1, o - 1], g[3, 5], x[n - 1, i - 1], x[3, 7] = 2.0, 3.0, 0.5, 4.0
    dw, db = layers().linear_weight_grad(g, x, bias=True)
    assert dw[o - 1, i - 1] == 1.0 and dw[5, 7] == 12.0 and int((dw != 0).sum()) == 2
    assert db[o - 1] == 2.0 and db[5] == 3.0 and int((db != 0).sum()) == 2
    w = torch.ones(o, i, dtype=torch.bfloat16, device="cuda")
    y = layers().linear(x, w, residual=g, out=g)
    assert (y[n - 1, : o - 1] == 0.5).all() and y[n - 1, o - 1] == 2.5 and (y[4] == 0).all()
