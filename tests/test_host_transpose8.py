"""transpose_8bit on host tensors: the values, in memory of their own, without
autograd's record."""
import pytest
import torch

from paper_2609_38767_amd import layers as m


def weight(o, i):
    g = torch.Generator().manual_seed(o + i)
    return (torch.randn(o, i, generator=g).to(torch.float8_e4m3fn), torch.rand(-(-o // 128), -(-i // 128), generator=g))


@pytest.mark.parametrize("o,i", [(1, 1), (1, 300), (300, 1), (200, 130), (129, 128)])
def test_the_transposed_weight_is_a_copy(o, i):
    q, s = weight(o, i)
    qt, st = m.transpose_8bit((q, s.requires_grad_()))
    assert torch.equal(qt.float(), q.float().t()) and torch.equal(st, s.t()) and not st.requires_grad
    assert qt.is_contiguous() and st.is_contiguous()
    assert qt.data_ptr() != q.data_ptr() and st.data_ptr() != s.data_ptr()
