"""The norm, 8-bit products and experts' products where offsets pass 32 bits and
where one grid dimension does not hold the threads."""
import pytest
import torch

pytestmark = pytest.mark.gpu
B = torch.bfloat16


def layers():
    from paper_2609_38767_amd import layers as m
    return m


def test_norm_of_more_than_2_to_32_elements():
    """Rows of one value each: y = sign, the gradient of a constant row's norm along itself 0; the last rows as the first."""
    n, d = 70000, 65536
    x = torch.ones(n, d, dtype=B, device="cuda")
    x[-1] = -3.0
    x[-2, :32768] = 2.0
    w = torch.ones(d, dtype=B, device="cuda")
    y = layers().rms_norm(x, w, eps=0.0)
    assert (y[0] == 1).all() and (y[35000] == 1).all() and (y[-1] == -1).all()
    want = layers().rms_norm(x[-3:].contiguous(), w, eps=0.0)
    assert torch.equal(y[-3:], want)
    del y
    q, s = layers().rms_norm_8bit(x, w, eps=0.0)
    assert (s[0] == 1 / torch.tensor(448.0)).all() and (q[-1].float() == -448).all() and (q[40000].float() == 448).all()
    q, s = layers().quantize_rows(x)
    want = torch.tensor(3.0) / torch.tensor(448.0)  # a division: 3 / tensor is a product with its reciprocal
    assert (q[-1].float() == -448).all() and (s[-1] == want).all()


def test_norm_gradient_of_more_than_2_to_32_elements():
    n, d = 300000, 16384
    h = torch.ones(n, d, dtype=B, device="cuda")
    h[-1, ::2] = 3.0
    w = torch.ones(d, dtype=B, device="cuda")
    g = torch.zeros(n, d, dtype=B, device="cuda")
    g[-1], g[0] = 1.0, 1.0
    out, dw = layers().rms_norm_grad(g, h, w, eps=0.0, out=None)
    want = layers().rms_norm_grad(g[-1:].contiguous(), h[-1:].contiguous(), w, eps=0.0)
    assert torch.equal(out[-1:], want[0]) and not out[0].any() and not out[150000].any()
    # row 0 adds 1 (h u = 1), row n - 1 what it adds alone
    assert torch.equal(dw, want[1] + 1)


@pytest.mark.parametrize("d", [8, 3])
def test_norm_of_many_short_rows(d):
    n = (1 << 26) + 5000
    x = torch.full((n, d), 2.0, dtype=B, device="cuda")
    x[-1] = -1.0
    y = layers().rms_norm(x, torch.ones(d, dtype=B, device="cuda"), eps=0.0)
    assert (y[:-1] == 1).all() and (y[-1] == -1).all()


def test_8bit_product_of_long_operands():
    """Rows, weights and results past 2^32 bytes."""
    n, i, o = 530000, 8208, 40
    x = torch.zeros(n, i, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    one = torch.tensor(1.0).to(torch.float8_e4m3fn).cuda()
    x[-1], x[0, :5] = one, one
    sx = torch.full((n, 65), 0.5, device="cuda")
    w8 = torch.ones(o, i, device="cuda").to(torch.float8_e4m3fn), torch.ones(1, 65, device="cuda")
    y = layers().linear_8bit((x, sx), w8)
    assert (y[-1] == 4104).all() and (y[0] == 2.5).all() and not y[1:-1].any()
    del y
    y = layers().linear_8bit((w8[0][:3], torch.ones(3, 65, device="cuda")), (x, torch.ones(-(-n // 128), 65, device="cuda")))
    assert y.shape == (3, n) and (y[:, -1] == 8192).all() and (y[:, 0] == 5).all() and not y[:, 1:-1].any()  # 8208 in bf16
    y = layers().linear_8bit((w8[0], torch.ones(o, 65, device="cuda")), (x, torch.ones(-(-n // 128), 65, device="cuda")))
    assert (y[:, -1] == 8192).all() and (y[:, 0] == 5).all() and not y[:, 1:-1].any()


def test_experts_of_long_weights():
    """Weights past 2^32 elements: the last expert's are met; its weight gradient lands in its place."""
    e, o, i = 70, 8192, 8192
    w = torch.zeros(e, o, i, dtype=B, device="cuda")
    w[-1] = 1.0
    off = torch.zeros(e + 1, dtype=torch.int64, device="cuda")
    off[-1] = 3
    x = torch.ones(4, i, dtype=B, device="cuda")
    y = layers().expert_linear(x, w, off)
    assert (y[:3] == 8192).all() and not y[3].any()
    d = layers().expert_linear_input_grad(x, w, off)
    assert (d[:3] == 8192).all() and not d[3].any()
    del w
    out = torch.full((e, o, i), 7.0, device="cuda")
    layers().expert_linear_weight_grad(x, x, off, out=out)
    assert (out[-1] == 3).all() and not out[:-1].any()


def test_experts_of_long_rows():
    """Rows past 2^31 elements, two experts that meet behind that."""
    n, i, o = 1 << 20, 4104, 16
    x = torch.zeros(n, i, dtype=B, device="cuda")
    x[-1], x[-3] = 1.0, 1.0
    w = torch.ones(2, o, i, dtype=B, device="cuda")
    w[1] *= 2
    off = torch.tensor([5, n - 2, n], device="cuda")
    y = layers().expert_linear(x, w, off)
    assert (y[-1] == 8192).all() and (y[-3] == 4096).all() and not y[:-3].any() and not y[-2].any()  # 8208, 4104 in bf16
    g = torch.zeros(n, o, dtype=B, device="cuda")
    g[-1], g[-3] = 1.0, 3.0
    dw, db = layers().expert_linear_weight_grad(g, x, off, bias=True)
    assert (dw[0] == 3).all() and (dw[1] == 1).all() and (db[0] == 3).all() and (db[1] == 1).all()
