"""Model-side operators over more rows than one grid dimension holds threads for:
a wave per row and 2^26 rows are 2^32 threads."""
import pytest
import torch

pytestmark = pytest.mark.gpu
N = (1 << 26) + 5000


def layers():
    from paper_2609_38767_amd import layers as m
    return m


@pytest.mark.parametrize("d,dtype", [(8, torch.bfloat16), (3, torch.float32)])
def test_lookup_of_many_tokens(d, dtype):
    table = torch.arange(1, 6, device="cuda")[:, None].expand(5, d).to(dtype).contiguous()
    t = (torch.arange(N, device="cuda") % 5).int()
    out = torch.full((N, d), -1.0, dtype=dtype, device="cuda")
    layers().embedding(table, t, out=out)
    assert torch.equal(out[:, 0], (t + 1).to(dtype)) and torch.equal(out[:, -1], out[:, 0])


def test_table_gradient_of_many_tokens():
    """Every position its own row, in falling order, so that the last places of the sort have rows of their own."""
    t = torch.arange(N - 1, -1, -1, device="cuda").int()
    g = (torch.arange(N, device="cuda") % 128).to(torch.bfloat16)[:, None].expand(N, 4).contiguous()
    out = torch.full((N, 4), -1.0, device="cuda")
    layers().embedding_grad(g, t, N, out=out)
    want = (torch.arange(N - 1, -1, -1, device="cuda") % 128).float()
    assert all(torch.equal(out[:, c], want) for c in range(4))


def test_product_of_many_repacked_rows():
    """Rows of three elements are repacked by a wave each; one of them has a value of its own at either end."""
    x = torch.ones(N, 3, dtype=torch.bfloat16, device="cuda")
    x[0, 2], x[N - 1, 0] = 3.0, 5.0
    w = torch.tensor([[1.0, 2.0, 4.0], [1.0, 0.0, 0.0]], dtype=torch.bfloat16, device="cuda")
    y = layers().linear(x, w)
    assert y[0].tolist() == [15.0, 1.0] and y[N - 1].tolist() == [11.0, 5.0]
    assert (y[1:N - 1, 0] == 7).all() and (y[1:N - 1, 1] == 1).all()
