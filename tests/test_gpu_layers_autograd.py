"""The example's autograd functions: first derivatives as the layers give them, second ones refused."""
import importlib.util
import os

import pytest
import torch

import layer_util as L

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_layers.py")
    spec = importlib.util.spec_from_file_location("packed_layers", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def layers():
    e = example()
    pos = L.positions(40, [[25, 15]])
    heads = [L.normal((1, 40, 2, 32), torch.bfloat16, s).requires_grad_() for s in range(3)]
    rows = [L.normal((1, 40, 16), torch.bfloat16, s).requires_grad_() for s in range(2)]
    inv = torch.ones(16, device=L.DEV)
    return {"rotary": (heads[:1], lambda: e.Rotary.apply(heads[0], pos, inv)),
            "attention": (heads, lambda: e.Attention.apply(*heads, pos, 30.0)),
            "recurrence": (rows, lambda: e.Recurrence.apply(*rows, pos))}


@pytest.mark.parametrize("name", ["rotary", "attention", "recurrence"])
def test_a_second_derivative_is_refused(name):
    inputs, run = layers()[name]
    dy = L.normal(run().shape, torch.bfloat16, 9).requires_grad_()
    first = torch.autograd.grad(run(), inputs, dy, create_graph=True)
    assert all(bool(torch.isfinite(g).all()) and bool(g.any()) for g in first)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        sum(g.float().square().sum() for g in first).backward()
