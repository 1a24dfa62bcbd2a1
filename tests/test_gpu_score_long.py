"""Scoring with more rows or queries than one grid dimension holds threads for:
2^26 rows of a wave each, 2^22 queries of 1024 threads each."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _score(*a, **kw):
    from paper_2609_38767_amd.session import score
    return score(*a, **kw)


@pytest.mark.parametrize("n_q,dtype,F", [(1, "f32", 8), (1, "bf16", 8), (20, "bf16", 32)])
def test_cosine_of_many_rows(n_q, dtype, F):
    """Rows and queries of ones but for one element: the cosine is known in closed form."""
    n = (1 << 26) + 5000
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    a = (torch.arange(n, device="cuda") % 3).float()
    x = torch.ones(n, F, dtype=dt, device="cuda")
    x[:, 1] = a.to(dt)
    S, _, _ = _score(torch.ones(n_q, F, dtype=dt, device="cuda"), x, cosine=True)
    want = (F - 1 + a) / ((F - 1 + a * a) * F).sqrt()
    # whole numbers in every sum: the norms' roots, their reciprocals and two products round
    assert ((S - want).abs() <= 16 * 2.0 ** -24 * want).all()


def test_top_k_of_many_queries():
    n_q = (1 << 22) + 100
    a = torch.arange(n_q, device="cuda")
    q = torch.zeros(n_q, 8, device="cuda")
    q[a, a % 8] = 1.0  # query i picks column i % 8 of the training rows
    t = torch.zeros(16, 8)
    t[torch.arange(8) + 8, torch.arange(8)] = torch.arange(1, 9).float()
    t = t.cuda()
    _, idx, val = _score(q, t, topk=2, want_scores=False)
    assert torch.equal(idx[:, 0].long(), 8 + a % 8) and torch.equal(val[:, 0], (a % 8 + 1).float())
    assert not idx[:, 1].any() and not val[:, 1].any()  # zeros: the lowest index
