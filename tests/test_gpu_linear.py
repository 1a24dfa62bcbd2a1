"""Linear layers with a fused epilogue and their backward products on the GPU
against the float64 oracle, elementwise within derived bounds."""
import numpy as np
import pytest
import torch

from model_util import DT, EVAL, OUT, SLOPE, U, check, gen, host, product_bound, rand
from oracle import model as om

pytestmark = pytest.mark.gpu

# rows, d_in, d_out: single rows and columns, tile edges and one off them, odd
# widths, few rows against wide layers, deep sums
SIZES = [(1, 1, 1), (1, 64, 32), (2, 8, 4096), (3, 33, 65), (5, 2049, 17), (7, 768, 2304), (16, 4096, 128),
         (17, 1000, 264), (33, 520, 72), (64, 64, 64), (65, 129, 257), (127, 256, 512), (128, 4104, 136), (200, 31, 1030),
         (255, 72, 8), (256, 512, 256), (257, 264, 520), (513, 128, 384), (1030, 200, 264), (300, 1, 300), (2051, 8, 24)]
DTYPES = ["f32", "bf16"]


def layers():
    from paper_2609_38767_amd import layers as m
    return m


def _forward_bound(x, w, z, y, kind, r, dtype):
    e = product_bound(x, w.T) + 2 * U * np.abs(z)
    bz = e + OUT[dtype] * (np.abs(z) + e)
    ey = SLOPE * e + EVAL * np.abs(z)
    by = ey + OUT[dtype] * (np.abs(y) + ey) + 2 * U * (np.abs(y) + (np.abs(r) if r is not None else 0))
    return by, bz


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(size, dtype):
    n, i, o = size
    k = SIZES.index(size)
    kind, g = om.ACTS[k % 5], gen(k)
    x, w = rand(g, n, i, dtype=dtype), rand(g, o, i, dtype=dtype, std=i ** -0.5)
    b = rand(g, o, dtype=dtype) if k % 3 else None
    r = rand(g, n, o, dtype=dtype) if k % 2 else None
    y, z = layers().linear(x, w, b, act=kind, residual=r, keep_preact=True)
    want, wz = om.linear(host(x), host(w), None if b is None else host(b), kind, None if r is None else host(r))
    by, bz = _forward_bound(host(x), host(w), wz, want, kind, None if r is None else host(r), dtype)
    check(z, wz, bz, "z")
    check(y, want, by, "y")
    again = layers().linear(x, w, b, act=kind, residual=r)
    assert torch.equal(again, y)  # the same bits, also without z


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_input_grad(size, dtype):
    n, i, o = size
    k = SIZES.index(size)
    kind, g = om.ACTS[(k + 1) % 5], gen(100 + k)
    gr, w = rand(g, n, o, dtype=dtype), rand(g, o, i, dtype=dtype, std=o ** -0.5)
    z = rand(g, n, i, dtype=dtype, std=2.0) if kind != "none" else None
    r = rand(g, n, i, dtype=dtype) if k % 2 else None
    d, p = layers().linear_input_grad(gr, w, residual=r, act=kind, preact=z, both=True)
    wd, wp = om.linear_input_grad(host(gr), host(w), None if r is None else host(r), kind,
                                  None if z is None else host(z))
    e = product_bound(host(gr), host(w)) + 2 * U * np.abs(wd)
    if r is not None:
        e = e + 2 * U * np.abs(host(r))
    check(d, wd, e + OUT[dtype] * (np.abs(wd) + e), "d")
    ep = SLOPE * e + EVAL * np.abs(wd) * (1 if z is None else 1 + np.abs(host(z)))
    check(p, wp, ep + OUT[dtype] * (np.abs(wp) + ep), "p")
    only = layers().linear_input_grad(gr, w, residual=r, act=kind, preact=z)
    assert torch.equal(only, p)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_weight_grad(size, dtype):
    n, i, o = size
    g = gen(200 + SIZES.index(size))
    gr, x = rand(g, n, o, dtype=dtype), rand(g, n, i, dtype=dtype)
    dw, db = layers().linear_weight_grad(gr, x, bias=True)
    ww, wb = om.linear_weight_grad(host(gr), host(x))
    bw = product_bound(host(gr).T, host(x))
    bb = 2 * (n + 8) * U * np.abs(host(gr)).sum(0)
    assert dw.dtype == db.dtype == torch.float32
    check(dw, ww, bw, "dw")
    check(db, wb, bb, "db")
    assert torch.equal(layers().linear_weight_grad(gr, x), dw)
    # accumulation adds to what is there: one more rounding of the sum
    w0, b0 = rand(g, o, i), rand(g, o)
    aw, ab = layers().linear_weight_grad(gr, x, bias=True, out=w0.clone(), out_bias=b0.clone(), accumulate=True)
    check(aw, ww + host(w0), bw + U * (np.abs(ww + host(w0)) + bw), "dw accumulated")
    check(ab, wb + host(b0), bb + U * (np.abs(wb + host(b0)) + bb), "db accumulated")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size,pad,offset", [((9, 40, 24), 8, 8), ((70, 136, 200), 3, 1), ((1, 257, 129), 5, 3),
                                             ((130, 64, 264), 1, 0), ((300, 520, 7), 0, 1)])
def test_strided_and_unaligned_rows(size, pad, offset, dtype):
    """Padded and misaligned operands whose surroundings are NaN; outputs in padded rows leave the padding alone."""
    n, i, o = size
    g = gen(17)
    x, w = rand(g, n, i, dtype=dtype, pad=pad, offset=offset), rand(g, o, i, dtype=dtype, pad=pad, offset=offset)
    r, b = rand(g, n, o, dtype=dtype, pad=pad, offset=offset), rand(g, o, dtype=dtype, offset=offset)
    out = torch.full((n, o + pad), 7.0, dtype=DT[dtype], device="cuda")
    layers().linear(x, w, b, act="relu", residual=r, out=out[:, :o])
    want, wz = om.linear(host(x), host(w), host(b), "relu", host(r))
    check(out[:, :o], want, _forward_bound(host(x), host(w), wz, want, "relu", host(r), dtype)[0])
    assert (out[:, o:] == 7).all()
    gr, z = rand(g, n, o, dtype=dtype, pad=pad, offset=offset), rand(g, n, i, dtype=dtype, pad=pad, offset=offset)
    q = rand(g, n, i, dtype=dtype, pad=pad, offset=offset)
    d = layers().linear_input_grad(gr, w, residual=q)
    wd, _ = om.linear_input_grad(host(gr), host(w), host(q))
    e = product_bound(host(gr), host(w)) + 2 * U * (np.abs(wd) + np.abs(host(q)))
    check(d, wd, e + OUT[dtype] * (np.abs(wd) + e))
    p = layers().linear_input_grad(gr, w, residual=q, act="relu", preact=z)
    assert torch.equal(p, torch.where(z <= 0, torch.zeros_like(d), d))
    dw, db = layers().linear_weight_grad(gr, x, bias=True)
    ww, wb = om.linear_weight_grad(host(gr), host(x))
    check(dw, ww, product_bound(host(gr).T, host(x)))
    check(db, wb, 2 * (n + 8) * U * np.abs(host(gr)).sum(0))


@pytest.mark.parametrize("dtype", DTYPES)
def test_in_place_and_leading_axes(dtype):
    g = gen(23)
    x, w, r = rand(g, 3, 50, 72, dtype=dtype), rand(g, 40, 72, dtype=dtype), rand(g, 3, 50, 40, dtype=dtype)
    want = layers().linear(x, w, residual=r)
    assert want.shape == (3, 50, 40)
    y = r.clone()
    assert layers().linear(x, w, residual=y, out=y) is y and torch.equal(y, want)
    z = rand(g, 3, 50, 72, dtype=dtype)
    want = layers().linear_input_grad(r, w, residual=x, act="silu", preact=z)
    d, p = x.clone(), z.clone()
    assert torch.equal(layers().linear_input_grad(r, w, residual=d, act="silu", preact=z, out=d), want)
    assert torch.equal(layers().linear_input_grad(r, w, residual=x, act="silu", preact=p, out=p), want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(dtype):
    g = gen(5)
    x, w = torch.empty(0, 24, dtype=DT[dtype], device="cuda"), rand(g, 16, 24, dtype=dtype)
    gr = torch.empty(0, 16, dtype=DT[dtype], device="cuda")
    assert layers().linear(x, w).shape == (0, 16)
    assert layers().linear_input_grad(gr, w).shape == (0, 24)
    dw, db = layers().linear_weight_grad(gr, x, bias=True)
    assert dw.shape == (16, 24) and not dw.any() and not db.any()
    dw.fill_(3)
    layers().linear_weight_grad(gr, x, out=dw, accumulate=True)
    assert (dw == 3).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(3, 72, 40), (130, 264, 520), (300, 200, 136)])
def test_non_finite_values_stay_where_they_are(size, dtype):
    """An infinity or NaN of one row or column reaches that row or column of the
    result only; all others are as without it."""
    n, i, o = size
    g = gen(31)
    x, w = rand(g, n, i, dtype=dtype), rand(g, o, i, dtype=dtype)
    clean = layers().linear(x, w)
    bad = x.clone()
    bad[n // 2, i // 3] = float("inf")
    bad[n - 1, i - 1] = float("nan")
    y = layers().linear(bad, w)
    keep = [k for k in range(n) if k not in (n // 2, n - 1)]
    assert torch.equal(y[keep], clean[keep])
    assert torch.isnan(y[n - 1]).all()
    assert torch.equal(torch.isposinf(y[n // 2]), w[:, i // 3] > 0)
    gr = rand(g, n, o, dtype=dtype)
    gr[:, o // 2] = float("nan")
    dw, db = layers().linear_weight_grad(gr, x, bias=True)
    assert torch.isnan(dw[o // 2]).all() and torch.isnan(db).nonzero().flatten().tolist() == [o // 2]
    assert torch.isfinite(dw[[k for k in range(o) if k != o // 2]]).all()


@pytest.mark.parametrize("kind", om.ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_activations_over_their_range(kind, dtype):
    """One column carries z through an identity weight: values, slopes, limits."""
    z = torch.cat([torch.linspace(-12, 12, 2001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 30.0, -30.0, 1e18, -1e18])])
    z = z.to(DT[dtype]).cuda()[:, None].contiguous()
    one = torch.ones(1, 1, dtype=DT[dtype], device="cuda")
    y = layers().linear(z, one, act=kind)
    h = host(z)
    with np.errstate(over="ignore"):
        want = om.act(h, kind)
    check(y, want, (EVAL + OUT[dtype]) * np.abs(h) * np.minimum(1, np.exp(-np.abs(h) * (h < 0)) * 64 + (h > 0)) +
          OUT[dtype] * np.abs(want) + 1e-38, "value")
    p = layers().linear_input_grad(torch.ones_like(z), one, act=kind, preact=z)
    small = np.abs(h) <= 40
    ws = om.act_slope(np.where(small, h, 0.0), kind)
    ws = np.where(small, ws, 1.0 if kind == "none" else (h > 0) * 1.0)
    # float32 evaluation: the argument's rounding enters the slope as |z| times the second derivative (<= 1)
    check(p, ws, OUT[dtype] * np.abs(ws) + EVAL * (1 + np.where(small, np.abs(h), 0)), "slope")


def test_infinite_preactivations_take_the_limits():
    inf = float("inf")
    z = torch.tensor([[inf], [-inf], [float("nan")]], device="cuda")
    one = torch.ones(1, 1, device="cuda")
    for kind in om.ACTS[1:]:
        y = layers().linear(z, one, act=kind).flatten().tolist()
        assert y[0] == inf and y[1] == 0 and y[2] != y[2], kind
        p = layers().linear_input_grad(torch.ones_like(z), one, act=kind, preact=z).flatten().tolist()
        assert p[:2] == [1, 0], kind


def test_gradient_by_differences():
    """The backward products in float32 against central differences of the
    float64 forward pass at the same values."""
    g = gen(41)
    n, i, o = 6, 10, 7
    x, w, b, c = rand(g, n, i), rand(g, o, i), rand(g, o), rand(g, n, o)
    _, z = layers().linear(x, w, b, act="gelu", keep_preact=True)
    h = 1e-6

    def loss(x, w, b):
        return float((host(c) * om.linear(x, w, b, "gelu")[0]).sum())

    # dL/dz through the epilogue of a product with the identity
    gz = layers().linear_input_grad(c, torch.eye(o, device="cuda"), act="gelu", preact=z)
    dx, (dw, db) = layers().linear_input_grad(gz, w), layers().linear_weight_grad(gz, x, bias=True)
    args = [host(x), host(w), host(b)]
    for k, got in enumerate((dx, dw, db)):
        want = np.zeros_like(args[k])
        for at in np.ndindex(want.shape):
            hi, lo = [a.copy() for a in args], [a.copy() for a in args]
            hi[k][at] += h
            lo[k][at] -= h
            want[at] = (loss(*hi) - loss(*lo)) / (2 * h)
        # float32 products of about ten terms of size one, and the difference's own 1e-8
        assert np.abs(host(got) - want).max() < 64 * 10 * U * 8 + 1e-7


def test_another_stream():
    g = gen(47)
    x, w = rand(g, 600, 520, dtype="bf16"), rand(g, 264, 520, dtype="bf16")
    want = layers().linear(x, w, act="silu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y = layers().linear(x, w, act="silu", stream=s)
    h = layers().linear(x, w, act="silu", stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(y, want) and torch.equal(h, want)


def test_refusals():
    m = layers()
    x, w = torch.zeros(4, 8, device="cuda"), torch.zeros(6, 8, device="cuda")
    for bad in (lambda: m.linear(x.cpu(), w), lambda: m.linear(x.half(), w.half()), lambda: m.linear(x, w.bfloat16()),
                lambda: m.linear(x[:, :7], w), lambda: m.linear(x, w, act="tanh"), lambda: m.linear(x.t(), w[:, :4]),
                lambda: m.linear(x, w, torch.zeros(5, device="cuda")), lambda: m.linear(x, w, residual=x),
                lambda: m.linear_input_grad(x[:, :6], w, act="relu"), lambda: m.linear_input_grad(x, w),
                lambda: m.linear_weight_grad(x, w), lambda: m.linear_weight_grad(x, x, accumulate=True),
                lambda: m.linear(x.expand(3, 4, 8)[:, ::2], w),
                lambda: m.linear(x, w, out=torch.zeros(4, 6, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 300])
def test_graph_replays(rows, dtype):
    """Captured calls give the eager bits at every replay."""
    g = gen(53)
    x, w, b = rand(g, rows, 520, dtype=dtype), rand(g, 264, 520, dtype=dtype), rand(g, 264, dtype=dtype)

    def step():
        y, z = layers().linear(x, w, b, act="gelu_tanh", keep_preact=True)
        return (y, layers().linear_input_grad(y, w, act="relu", preact=x), *layers().linear_weight_grad(y, x, bias=True))

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        x.copy_(rand(g, rows, 520, dtype=dtype))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), k
