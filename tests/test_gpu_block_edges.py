"""Norms, 8-bit rows and products and experts' products at the ends of what their
entry points take: the smallest scales, the most rows, experts that nothing meets,
operands and outputs off their usual alignment."""
import numpy as np
import pytest
import torch

from expert_cuts import BIG, FEW, PADDED
from model_util import DT, OUT, U, check, gen, host, product_bound, rand
from oracle import block as ob

pytestmark = pytest.mark.gpu
DTYPES = ["f32", "bf16"]


def layers():
    from paper_2609_38767_amd import layers as m
    return m


# ------------------------------------------------------ 8-bit values under small scales
def halves(m, e):
    """A group whose scale is m 2^e, as near as its largest value says: 448 scales, every value halfway between two e4m3
    values, as near as float32 comes, and zero."""
    values = sorted({(8 + k) * 2.0 ** (x - 3) for x in range(-6, 9) for k in range(8) if (8 + k) * 2.0 ** (x - 3) <= 448}
                    | {k * 2.0 ** -9 for k in range(8)})
    ties = [(a + b) / 2 for a, b in zip(values, values[1:])]
    assert len(ties) == 126
    signs = np.where(np.arange(126) % 3 == 0, -1.0, 1.0)
    return np.concatenate([[448.0], np.array(ties) * signs, [0.0]]) * m * 2.0 ** e


def groups(dtype):
    rng = np.random.default_rng(2)
    m = [1.0, 1.25, 1.5, 1.75] + ([] if dtype == "bf16" else list(1 + rng.integers(0, 1 << 23, 4) * 2.0 ** -23))
    return np.stack([halves(v, e) for e in range(-128, -56) for v in m]).astype(np.float32)


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_under_small_scales(dtype):
    """The very values of the definition down to the smallest scale, at quotients that a wrong last bit moves."""
    m = layers()
    x = torch.from_numpy(groups(dtype)).to(DT[dtype]).cuda()
    q, s = m.quantize_rows(x)
    wq, ws = ob.quantize(host(x))
    assert np.array_equal(host(s), ws) and np.array_equal(host(q), wq)
    w = x[::16].repeat_interleave(128, 0)  # blocks of one scale
    q, s = m.quantize_weight(w)
    wq, ws = ob.quantize(host(w), 128)
    assert np.array_equal(host(s), ws) and np.array_equal(host(q), wq)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,d", [(3, 128), (2, 4096), (2, 4001), (2, 33024), (2, 66048), (2, 70001), (2049, 1001)])
def test_norms_under_small_scales(n, d, dtype):
    """Rows of ones, whose norm is the weight itself: every form that writes 8-bit rows."""
    m = layers()
    w = torch.from_numpy(np.resize(groups(dtype).reshape(-1)[::-1], d).copy()).to(DT[dtype]).cuda()
    (q, s), y = m.rms_norm_8bit(torch.ones(n, d, dtype=DT[dtype], device="cuda"), w, eps=0.0, keep=True)
    assert torch.equal(y, w.expand(n, d))
    wq, ws = ob.quantize(host(w)[None])
    assert np.array_equal(host(s), np.repeat(ws, n, 0)) and np.array_equal(host(q), np.repeat(wq, n, 0))


# ------------------------------------------------------ experts
def test_experts_of_the_most_rows():
    """One expert of all rows but one, as many as a call takes: every row is written, the last one too."""
    m, n = layers(), (1 << 31) - 1
    off = torch.tensor([0, 1, n], device="cuda")
    x = torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    x[0], x[1], x[-40], x[-1] = 1.0, 2.0, 3.0, 4.0
    w = torch.ones(2, 1, 8, dtype=torch.bfloat16, device="cuda")
    w[1] = 2.0
    y = torch.full((n, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    m.expert_linear(x, w, off, out=y)
    assert [float(y[k]) for k in (0, 1, -40, -1)] == [8, 32, 48, 64] and int(y.count_nonzero()) == 4
    y.fill_(7.0)
    m.expert_linear_input_grad(x, w.view(2, 8, 1), off, out=y)
    assert [float(y[k]) for k in (0, 1, -40, -1)] == [8, 32, 48, 64] and int(y.count_nonzero()) == 4


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 6, 300])
def test_weights_that_nothing_meets_stay_where_they_are(rows, dtype):
    """Widths off 16 bytes are repacked into the workspace, of the weights only those of experts with rows.  All else is
    NaN, before and after: the other experts' weights and the workspace."""
    import paper_2609_38767_amd as dt
    m, g, e, i, o = layers(), gen(rows), 40, 203, 101
    f = [0] * 9 + [rows // 3] * 20 + [rows] * (e + 1 - 29)  # experts 8 and 28, of one row the latter alone
    off = torch.tensor(f, dtype=torch.int32, device="cuda")
    met = [k for k in range(e) if f[k] < f[k + 1]]
    w = torch.full((e, o, i), float("nan"), dtype=DT[dtype], device="cuda")
    for k in met:
        w[k] = rand(g, o, i, dtype=dtype, std=0.1)
    x, gr = rand(g, rows, i, dtype=dtype), rand(g, rows, o, dtype=dtype)
    code = dt.DATTRI_F32 if dtype == "f32" else dt.DATTRI_BF16
    size = w.element_size()
    for op, a, shape in ((dt.DATTRI_LINEAR_FORWARD, x, (rows, o)), (dt.DATTRI_LINEAR_INPUT_GRAD, gr, (rows, i))):
        n = dt.dattri_expert_linear_workspace_bytes(op, rows, e, i, o, code, False)
        ws, y = torch.full((n,), 255, dtype=torch.uint8, device="cuda"), torch.empty(shape, dtype=DT[dtype], device="cuda")
        if op == dt.DATTRI_LINEAR_FORWARD:
            dt.dattri_expert_linear(a, 0, w, 0, None, off, 4, dt.DATTRI_ACT_NONE, None, 0, y, 0, None, 0, rows, e, i, o, code,
                                    ws, n)
            want, hw = ob.expert_linear(host(a), host(w), f)[0], [host(w[k]).T for k in range(e)]
        else:
            dt.dattri_expert_linear_input_grad(a, 0, w, 0, off, 4, None, 0, dt.DATTRI_ACT_NONE, None, 0, None, 0, y, 0, rows, e,
                                               i, o, code, ws, n)
            want, hw = ob.expert_input_grad(host(a), host(w), f)[0], [host(w[k]) for k in range(e)]
        for k in met:
            s = slice(f[k], f[k + 1])
            b = product_bound(host(a[s]), hw[k])
            check(y[s], want[s], b + OUT[dtype] * (np.abs(want[s]) + b), (op, k))
        wide = -(-i * size // 16) * 16  # of a packed row of the weights
        assert int((ws != 255).sum()) <= n - (e - len(met)) * o * wide


@pytest.mark.parametrize("dtype", DTYPES)
def test_other_experts_are_met_in_a_replay(dtype):
    """Widths off 16 bytes in a captured graph whose boundaries and weights change: what is repacked follows them."""
    m, g = layers(), gen(77)
    n, e, i, o = 60, 12, 203, 101
    x, gr, w = rand(g, n, i, dtype=dtype), rand(g, n, o, dtype=dtype), rand(g, e, o, i, dtype=dtype, std=0.1)
    off = torch.zeros(e + 1, dtype=torch.int64, device="cuda")

    def run():
        return m.expert_linear(x, w, off), m.expert_linear_input_grad(gr, w, off)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for f in ([0] + [30] * 6 + [60] * 6, [0] * 8 + [1] + [60] * 4, list(range(0, 61, 5)), [0] * 13):
        off.copy_(torch.tensor(f))
        w.mul_(-0.75)
        graph.replay()
        want = run()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), f
        for k, at in ob.expert_rows(f, n):
            for y, a, b in ((want[0], x, w.transpose(1, 2)), (want[1], gr, w)):
                if k is None:
                    assert not y[at].any()
                else:
                    e64 = product_bound(host(a[at]), host(b[k]))
                    check(y[at], host(a[at]) @ host(b[k]), e64 + OUT[dtype] * (np.abs(host(a[at]) @ host(b[k])) + e64), (f, k))


def off_by_one(t):
    """t's values, dense, one element behind a place on 16 bytes."""
    flat = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape)
    flat.view(torch.uint8 if t.element_size() == 1 else t.dtype).copy_(t.view(torch.uint8) if t.element_size() == 1 else t)
    assert flat.data_ptr() % 16 != 0
    return flat


def packed(t):
    return t.numel() // t.shape[-1] * (-(-t.shape[-1] * t.element_size() // 16) * 16)


@pytest.mark.parametrize("which", [0, 1], ids=["rows", "weights"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n", [1, 70, 700])
def test_only_the_operand_off_16_bytes_is_repacked(n, dtype, which):
    """The other one is read where it is: its part of the workspace stays as it was, and the results are the same bits."""
    import paper_2609_38767_amd as dt
    m, g, e, i, o = layers(), gen(n + which), 5, 208, 112
    code, t = dt.DATTRI_F32 if dtype == "f32" else dt.DATTRI_BF16, DT[dtype]
    f = [0, n // 3, n // 3, n // 2, n, n]
    off = torch.tensor(f, dtype=torch.int32, device="cuda")
    x, gr, w = rand(g, n, i, dtype=dtype), rand(g, n, o, dtype=dtype), rand(g, e, o, i, dtype=dtype, std=0.1)
    (x8, sx), (w8, sw) = m.quantize_rows(x), m.quantize_weight(w[0])

    def room(need):
        return torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    none = dt.DATTRI_ACT_NONE
    for op, a, b, want in (("fwd", x, w, m.expert_linear(x, w, off)), ("in", gr, w, m.expert_linear_input_grad(gr, w, off)),
                           ("wgt", gr, x, m.expert_linear_weight_grad(gr, x, off)), ("8", x8, w8, m.linear_8bit((x8, sx), (w8, sw), dtype=t))):
        if which:
            b = off_by_one(b)
        else:
            a = off_by_one(a)
        y = torch.full_like(want, float("nan"))
        if op == "8":
            need = dt.dattri_linear_scaled_workspace_bytes(n, i, o, code, False)
            ws = room(need)
            dt.dattri_linear_scaled(a, 0, sx, 0, b, 0, sw, 0, None, none, None, 0, y, 0, None, 0, n, i, o, code, ws, need)
        else:
            need = dt.dattri_expert_linear_workspace_bytes(("fwd", "in", "wgt").index(op), n, e, i, o, code, False)
            ws = room(need)
            if op == "fwd":
                dt.dattri_expert_linear(a, 0, b, 0, None, off, 4, none, None, 0, y, 0, None, 0, n, e, i, o, code, ws, need)
            elif op == "in":
                dt.dattri_expert_linear_input_grad(a, 0, b, 0, off, 4, None, 0, none, None, 0, None, 0, y, 0, n, e, i, o, code,
                                                   ws, need)
            else:
                dt.dattri_expert_linear_weight_grad(a, 0, b, 0, off, 4, y, 0, None, False, n, e, i, o, code, ws, need)
        assert torch.equal(y, want), op
        assert int((ws != 255).sum()) <= need - packed(a if which else b), op


def boundaries(n, e, seed):
    """e experts of very different sizes, every seventh one empty, rows of no expert at both ends."""
    rng = np.random.default_rng(seed)
    share = rng.exponential(1.0, e) * (np.arange(e) % 7 != 3)
    at = n // 50 + np.concatenate([[0.0], np.cumsum(share / share.sum())]) * (n - n // 50 - n // 70)
    return [int(v) for v in at]


def product(op, dtype, n, e, i, o, f, g):
    """A product over rows with its residual, checked expert by expert (float64 products on the GPU)."""
    m = layers()
    off = torch.tensor(f, dtype=torch.int32, device="cuda")
    a, w = rand(g, n, i if op == 0 else o, dtype=dtype), rand(g, e, o, i, dtype=dtype, std=0.1)
    r = rand(g, n, o if op == 0 else i, dtype=dtype)
    got = m.expert_linear(a, w, off, residual=r) if op == 0 else m.expert_linear_input_grad(a, w, off, residual=r)
    for q, s in ob.expert_rows(f, n):
        want, b = r[s].double(), 2 * U * r[s].double().abs()
        if q is not None and s.stop > s.start:
            x, y = a[s].double(), (w[q].double().t() if op == 0 else w[q].double()).contiguous()
            b = b + 2 * (x.shape[1] + 8) * U * (x.abs() @ y.abs())
            want = want + x @ y
        b = b + 2 * U * want.abs()
        assert ((got[s].double() - want).abs() <= b + OUT[dtype] * (want.abs() + b)).all(), (q, s)


@pytest.mark.parametrize("case", FEW, ids=lambda c: "-".join(map(str, c)))
def test_few_rows_split_in_two(case):
    op, dtype, n, e, i, o, _ = case
    f = boundaries(n, e, FEW.index(case))
    product(op, dtype, n, e, i, o, f, gen(FEW.index(case)))


@pytest.mark.parametrize("case", BIG, ids=lambda c: "-".join(map(str, c)))
def test_largest_tiles_of_many_experts(case):
    """Tile rows, whole and half ones, of segments behind the first 64."""
    op, dtype, n, e, i, o = case
    f = boundaries(n, e, BIG.index(case))
    left = {(b - a) % 256 for a, b in zip(f[62:], f[63:])}
    assert any(0 < v <= 128 for v in left) and any(v > 128 for v in left)
    product(op, dtype, n, e, i, o, f, gen(50 + BIG.index(case)))


def test_boundaries_out_of_order_in_the_largest_tiles():
    """Offsets that no caller should pass: whatever comes out, nothing outside the outputs is written."""
    m, g = layers(), gen(60)
    _, dtype, n, e, i, o = BIG[0]
    f = torch.tensor(boundaries(n, e, 0))
    rng = torch.Generator().manual_seed(1)
    x, w, gr = rand(g, n, i, dtype=dtype), rand(g, e, o, i, dtype=dtype), rand(g, n, i, dtype=dtype)
    wt = rand(g, e, i, o, dtype=dtype)
    for off in (f.flip(0), f[torch.randperm(e + 1, generator=rng)], torch.tensor([0, n] * (e // 2) + [0]),
                f * 1000003 - n, torch.full((e + 1,), 1 << 40), f - (1 << 40)):
        off = off.cuda()
        out = torch.full((n + 2, o), 7.0, dtype=DT[dtype], device="cuda")
        m.expert_linear(x, w, off, out=out[1:-1])
        assert (out[0] == 7).all() and (out[-1] == 7).all()
        out.fill_(7.0)
        m.expert_linear_input_grad(gr, wt, off, out=out[1:-1])
        assert (out[0] == 7).all() and (out[-1] == 7).all()


@pytest.mark.parametrize("pad", [3, 4])
@pytest.mark.parametrize("case", PADDED, ids=lambda c: "-".join(map(str, c)))
def test_padded_weight_gradients(case, pad):
    """As the dense gradient, bit for bit; what lies between its rows stays."""
    dtype, n, e, i, o, _, _ = case
    m, g = layers(), gen(n + pad)
    f = boundaries(n, e, n)
    off = torch.tensor(f, device="cuda")
    gr, x = rand(g, n, o, dtype=dtype), rand(g, n, i, dtype=dtype)
    dense = m.expert_linear_weight_grad(gr, x, off)
    wide = torch.full((e * o, i + pad), 7.0, device="cuda")
    out = wide[:, :i].unflatten(0, (e, o))
    assert m.expert_linear_weight_grad(gr, x, off, out=out) is out
    assert torch.equal(out, dense) and (wide[:, i:] == 7).all()
    w0 = rand(g, e, o, i)
    dense, out[:] = w0.clone(), w0
    m.expert_linear_weight_grad(gr, x, off, out=dense, accumulate=True)
    m.expert_linear_weight_grad(gr, x, off, out=out, accumulate=True)
    assert torch.equal(out, dense) and (wide[:, i:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,e,i,o,offset", [(300, 4, 203, 96, 0), (5000, 2, 203, 101, 1), (0, 3, 9, 16, 0)])
def test_bias_gradients_alone(n, e, i, o, offset, dtype):
    """Without a weight gradient there are no operands of a product: the workspace of aligned ones is enough."""
    import paper_2609_38767_amd as dt
    g, code = gen(n + i), dt.DATTRI_F32 if dtype == "f32" else dt.DATTRI_BF16
    gr = rand(g, n, o, dtype=dtype, offset=offset)
    f = boundaries(n, e, n)
    off = torch.tensor(f, device="cuda")
    want = np.stack([host(gr[s]).sum(0) for k, s in ob.expert_rows(f, n) if k is not None])
    bound = 2 * (n + 8) * U * np.stack([np.abs(host(gr[s])).sum(0) for k, s in ob.expert_rows(f, n) if k is not None])
    db = torch.full((e, o), 7.0, device="cuda")
    need = dt.dattri_expert_linear_workspace_bytes(dt.DATTRI_LINEAR_WEIGHT_GRAD, n, e, i, o, code, True)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dt.dattri_expert_linear_weight_grad(gr, 0, None, 0, off, 8, None, 0, db, False, n, e, i, o, code, ws, need)
    check(db, want, bound)
    db = torch.full((o,), 7.0, device="cuda")
    need = dt.dattri_linear_workspace_bytes(dt.DATTRI_LINEAR_WEIGHT_GRAD, n, i, o, code, True)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dt.dattri_linear_weight_grad(gr, 0, None, 0, None, 0, db, False, n, i, o, code, ws, need)
    check(db, host(gr).sum(0), 2 * (n + 8) * U * np.abs(host(gr)).sum(0))


# ------------------------------------------------------ strides of 8-bit outputs
class Padded:
    """Bytes and scales in padded rows, `offset` bytes into their buffer; all of it 0xA5 (and 7) at first."""

    def __init__(self, n, srows, d, offset, pad, spad):
        k = -(-d // 128)
        self.bytes = torch.full((offset + n * (d + pad) + 8,), 0xA5, dtype=torch.uint8, device="cuda")
        self.q = self.bytes[offset:offset + n * (d + pad)].view(n, d + pad)
        self.s = torch.full((srows + 1, k + spad), 7.0, device="cuda")
        self.n, self.d, self.k, self.offset = n, d, k, offset
        self.ld_q, self.ld_s = d + pad, k + spad

    def holds(self, q, s):
        """The values and scales of the oracle, and nothing else was written."""
        assert np.array_equal(host(self.s[:-1, :self.k]), s)
        assert np.array_equal(host(self.q[:, :self.d].contiguous().view(torch.float8_e4m3fn)), q)
        assert (self.q[:, self.d:] == 0xA5).all() and (self.bytes[:self.offset] == 0xA5).all()
        assert (self.bytes[-8:] == 0xA5).all() and (self.s[-1] == 7).all() and (self.s[:, self.k:] == 7).all()


PLACES = [(0, 0, 1), (1, 3, 0), (4, 4, 2), (8, 8, 1), (2, 16, 3)]  # offset and padding of the bytes, padding of the scales


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset,pad,spad", PLACES)
@pytest.mark.parametrize("n,d", [(1, 1), (9, 64), (5, 128), (33, 264), (3, 769), (2049, 513), (130, 1024), (3, 4096), (2, 33024),
                                 (2, 66048), (2, 70001)])
def test_strides_of_8bit_rows(n, d, offset, pad, spad, dtype):
    """The norm of rows of +-1, which is +-w (the sums are whole numbers, their mean 1), and quantize_rows of it."""
    import paper_2609_38767_amd as dt
    g, code = gen(d + offset), dt.DATTRI_F32 if dtype == "f32" else dt.DATTRI_BF16
    w = rand(g, d, dtype=dtype)
    x = (torch.randint(0, 2, (n, 1), generator=g, device="cuda") * 2 - 1).to(DT[dtype]).expand(n, d).contiguous()
    y = x * w
    want = ob.quantize(host(y))
    p = Padded(n, n, d, offset, pad, spad)
    dt.dattri_rms_norm(x, 0, None, 0, w, 0.0, None, 0, None, 0, p.q, p.ld_q, p.s, p.ld_s, n, d, code)
    p.holds(*want)
    p = Padded(n, n, d, offset, pad, spad)
    dt.dattri_quantize_rows(y, 0, n, d, code, p.q, p.ld_q, p.s, p.ld_s)
    p.holds(*want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset,pad,spad", PLACES)
@pytest.mark.parametrize("o,i", [(1, 1), (128, 128), (129, 300), (300, 1040)])
def test_strides_of_8bit_weights(o, i, offset, pad, spad, dtype):
    import paper_2609_38767_amd as dt
    g, code = gen(o + offset), dt.DATTRI_F32 if dtype == "f32" else dt.DATTRI_BF16
    w = rand(g, o, i, dtype=dtype)
    p = Padded(o, -(-o // 128), i, offset, pad, spad)
    dt.dattri_quantize_weight(w, 0, o, i, code, p.q, p.ld_q, p.s, p.ld_s)
    p.holds(*ob.quantize(host(w), 128))


# ------------------------------------------------------ the transposed weight
@pytest.mark.parametrize("o,i", [(1, 200), (300, 1), (264, 520)])
def test_transposed_weight_on_a_stream_and_in_a_graph(o, i):
    m, g = layers(), gen(o)
    q, s = m.quantize_weight(rand(g, o, i))
    want = q.view(torch.uint8).t().clone(), s.t().clone()

    def same(w):
        return torch.equal(w[0].view(torch.uint8), want[0]) and torch.equal(w[1], want[1]) and w[0].is_contiguous()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [m.transpose_8bit((q, s), stream=v) for v in (side, side.cuda_stream, 0)]
    torch.cuda.synchronize()
    assert all(same(w) for w in got)
    with pytest.raises(ValueError, match="on the GPU"):
        m.transpose_8bit((q, s.cpu()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w = m.transpose_8bit((q, s))
    for k in range(3):
        q.view(torch.uint8).bitwise_xor_(k + 1)
        s.mul_(2)
        want = q.view(torch.uint8).t().clone(), s.t().clone()
        graph.replay()
        assert same(w)
