"""The examples' rotary positions under autograd with gradients as autograd hands them over: broadcast, or transposed."""
import importlib.util
import os

import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu


def example(name):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", name + ".py")
    spec = importlib.util.spec_from_file_location(name, path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("name", ["packed_layers", "packed_state_space"])
def test_gradients_that_are_broadcast_or_transposed(name):
    e, t, n = example(name), 40, 8
    pos, inv = L.positions(t, [[30, 10]]), torch.rand(n, device=L.DEV)
    coords, axis = torch.stack((pos, pos // 2)), (torch.arange(n, device=L.DEV) % 2).to(torch.int32)
    x = L.normal((1, t, 2, 2 * n), torch.float32, 1).requires_grad_()

    def turned():
        return e.Rotary.apply(x, pos, inv) if name == "packed_layers" else e.RotaryAxes.apply(x, pos, coords, axis, inv)

    def gradient(dy):
        dx = torch.empty_like(dy)
        if name == "packed_layers":
            B.bload_rotary_grad(pos, dy, dx, inv)
        else:
            B.bload_rotary_axes_grad(pos, coords, axis, dy, dx, inv)
        return dx

    got, = torch.autograd.grad(turned().sum(), x)  # (one number for all elements, all strides 0)
    assert torch.equal(got, gradient(torch.ones_like(x)))
    w = L.normal((1, t, 2 * n, 2), torch.float32, 2)
    got, = torch.autograd.grad((turned().transpose(2, 3) * w).sum(), x)
    assert torch.equal(got, gradient(w.transpose(2, 3).contiguous()))
