"""transpose_8bit on host tensors: the values, in memory of their own, without
autograd's record; what it refuses."""
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


def test_refusals():
    q, s = weight(200, 130)
    for bad in ((q.float(), s), (q, s[:1]), (q[None], s)):
        with pytest.raises(ValueError, match="128 x 128"):
            m.transpose_8bit(bad)
    with pytest.raises(ValueError, match="on the GPU"):  # a stream has nothing to do for host tensors
        m.transpose_8bit((q, s), stream=0)
