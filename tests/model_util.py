"""Inputs and error bounds shared by the tests of the model-side operators.

U is the unit roundoff of float32.  A float32 sum of K products in any order is
off by at most (K + 1) U sum |a b| to first order (each of K - 1 additions and
the product's own rounding); 2 (K + 8) U sum |a b| also covers the higher orders,
the joins of split sums, bias and residual.  A result of magnitude v is then
rounded to its type, by at most half a step: U v for float32 (24 significant
bits), 2^-8 v for bfloat16 (8 significant bits)."""
import numpy as np
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
OUT = {"f32": U, "bf16": 2.0 ** -8}
# |act'| <= 1.13 for all activations; float32 evaluation of act and act' (exp, erfc,
# reciprocal, the products around them) is within 32 U of max(|value|, 1 for slopes)
SLOPE, EVAL = 1.13, 32 * U


def host(t):
    return t.detach().to("cpu", torch.float64).numpy()


def product_bound(a, b):
    """Bound on a float32 product a @ b (float64 host arrays)."""
    return 2 * (a.shape[1] + 8) * U * (np.abs(a) @ np.abs(b))


def check(got, want, bound, what=""):
    got = host(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.abs(got - want).max()))


def rand(gen, *shape, dtype="f32", std=1.0, pad=0, offset=0):
    """A [.., d] tensor whose rows are d + pad apart, `offset` elements into its
    buffer; what lies around the rows is NaN, so a kernel that reads it shows."""
    n = int(np.prod(shape[:-1])) if len(shape) > 1 else 1
    d = shape[-1]
    buf = torch.full((offset + n * (d + pad) + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    t = buf[offset:offset + n * (d + pad)].view(n, d + pad)[:, :d]
    t.copy_((torch.randn(n, d, generator=gen, device="cuda") * std).to(DT[dtype]))
    return t.view(*shape[:-1], d) if pad == 0 else t if len(shape) == 2 else t.unflatten(0, shape[:-1])


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g
