"""Every way that the 8-bit products and the experts' products are cut, against
float64 products within the bounds of their own tests."""
import numpy as np
import pytest
import torch

from block_cuts import CUTS8, CUTSX
from model_util import DT, OUT, U, check, gen, host, rand
from oracle import block as ob

pytestmark = pytest.mark.gpu


def layers():
    from paper_2609_38767_amd import layers as m
    return m


def matmul64(a, b):
    """Float64 product of host matrices (on the GPU: some have 10^10 terms)."""
    return (torch.from_numpy(a).cuda() @ torch.from_numpy(np.ascontiguousarray(b)).cuda()).cpu().numpy()


def bound64(a, b):
    return 2 * (a.shape[1] + 8) * U * matmul64(np.abs(a), np.abs(b))


def eight(t, rows):
    q, s = ob.quantize(host(t), rows)
    return (torch.from_numpy(q).float().to(torch.float8_e4m3fn).cuda(), torch.from_numpy(s).cuda()), \
        q * ob.spread(s, *q.shape, rows)


def largest(v):
    return np.maximum.reduceat(np.abs(v), np.arange(0, v.shape[1], 8), axis=1)


@pytest.mark.parametrize("cut", CUTS8, ids=lambda c: "-".join(map(str, c)))
def test_8bit_products(cut):
    dtype, n, i, o, _, _ = cut
    g = gen(CUTS8.index(cut))
    x8, x = eight(rand(g, n, i) * torch.exp(rand(g, n, 1)), 1)
    w8, w = eight(rand(g, o, i, std=i ** -0.5), 128)
    b, r = rand(g, o, dtype=dtype), rand(g, n, o, dtype=dtype)
    y, z = layers().linear_8bit(x8, w8, b, residual=r, keep_preact=True, dtype=DT[dtype])
    want = matmul64(x, w.T) + host(b)
    e = bound64(x, w.T) + 8 * U * matmul64(np.abs(x), np.abs(w.T)) + 2 * U * np.abs(want)
    if dtype == "bf16":  # as derived beside the 8-bit products' tests
        e = e + 7 * 2.0 ** -13 * matmul64(largest(x), largest(w).T)
    check(z, want, e + OUT[dtype] * (np.abs(want) + e), "z")
    check(y, want + host(r), e + OUT[dtype] * (np.abs(want + host(r)) + e) + 2 * U * (np.abs(want) + np.abs(host(r))), "y")
    assert torch.equal(layers().linear_8bit(x8, w8, b, residual=r, dtype=DT[dtype]), y)


def boundaries(n, e, seed):
    """e experts of very different sizes, rows of no expert at both ends where there are many."""
    rng = np.random.default_rng(seed)
    a, b = (n // 50, n - n // 70) if n > 100 else (0, n)
    inner = np.sort(rng.integers(a, b + 1, e - 1)) if e > 1 else []
    return [a, *map(int, inner), b]


@pytest.mark.parametrize("cut", CUTSX, ids=lambda c: "-".join(map(str, c)))
def test_expert_products(cut):
    op, dtype, n, e, i, o, _, _ = cut
    k = CUTSX.index(cut)
    g, f = gen(50 + k), boundaries(n, e, k)
    off = torch.tensor(f, dtype=torch.int32, device="cuda")
    at = ob.expert_rows(f, n)
    if op == 2:
        gr, x = rand(g, n, o, dtype=dtype), rand(g, n, i, dtype=dtype)
        dw, db = layers().expert_linear_weight_grad(gr, x, off, bias=True)
        twice = dw.clone()
        layers().expert_linear_weight_grad(gr, x, off, out=twice, accumulate=True)
        assert torch.equal(twice, 2 * dw)
        for q, s in at:
            if q is not None:
                a, c = host(gr[s]), host(x[s])
                check(dw[q], matmul64(a.T.copy(), c), bound64(a.T.copy(), c), f"dw {q}")
                check(db[q], a.sum(0), 2 * (len(a) + 8) * U * np.abs(a).sum(0), f"db {q}")
        return
    a, w = rand(g, n, i if op == 0 else o, dtype=dtype), rand(g, e, o, i, dtype=dtype, std=0.1)
    wide = o if op == 0 else i
    r, b = rand(g, n, wide, dtype=dtype), rand(g, e, o, dtype=dtype)
    if op == 0:
        got = layers().expert_linear(a, w, off, b, residual=r)
    else:
        got = layers().expert_linear_input_grad(a, w, off, residual=r)
    want, bound = np.zeros((n, wide)), np.zeros((n, wide))
    for q, s in at:
        if q is not None:
            m = host(w[q]).T.copy() if op == 0 else host(w[q])
            want[s], bound[s] = matmul64(host(a[s]), m), bound64(host(a[s]), m)
            if op == 0:
                want[s] += host(b[q])
    bound = bound + 2 * U * (np.abs(want) + np.abs(host(r)))
    want = want + host(r)
    check(got, want, bound + OUT[dtype] * (np.abs(want) + bound))
