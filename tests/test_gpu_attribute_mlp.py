"""The example that trains with the model-side operators and attributes by
capture of the same pass: it learns, its gradients are those of torch's autograd
in float64, and the training sequences it names share the query's topic."""
import importlib.util
import os

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location("attribute_mlp", os.path.join(ROOT, "examples", "attribute_mlp.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_example_learns_and_attributes(dtype):
    losses, hits = _example().main(["--steps", "30", "--dtype", dtype])
    assert losses[-1] < losses[0] - 0.5  # it fits its few cycles
    assert hits > 0.5  # 1/8 by chance


def test_gradients_match_autograd_in_float64():
    m = _example()
    model = m.Model(97, 24, 40, 2, torch.float32)
    data, _ = m.sequences(6, 9, 97, 3, seed=5)
    x, y = data[:, :-1].contiguous(), data[:, 1:]
    logits, kept = model.forward(x)
    _, g = m.loss_and_gradient(logits, y)
    _, grads = model.backward(g, kept, x)
    w = {k: v.double().requires_grad_() for k, v in model.master.items()}
    h = w["table"][x] * model.scale
    for b in range(model.blocks):
        u = torch.nn.functional.gelu(h @ w[f"up{b}"].mT.contiguous() + w[f"up{b}.bias"])
        h = u @ w[f"down{b}"].mT.contiguous() + h
    torch.nn.functional.cross_entropy((h @ w["out"].mT.contiguous()).flatten(0, 1), y.flatten(), reduction="sum").backward()
    for k, v in grads.items():
        want = w[k].grad
        # float32 throughout: five products of sums of at most 97 terms, rounded at 2^-24 each
        assert (v.double() - want).norm() <= 1e-5 * want.norm(), k
