"""bload_scan and its gradient on long sequences that are walked in segments: what crosses from segment to segment where the product of a
segment's decays is beyond the range of 32 bits."""
import math

import pytest
import torch

import layer_util as L
import state_space_util as S
from test_gpu_scan import F32, call, compare

pytestmark = pytest.mark.gpu


def test_a_state_of_zero_stays_zero_whatever_grows():
    """Growing states (a > 0), inputs in the last 46 slots and gradients in the first 60 only: in between there is nothing to grow, by
    exp(0.4 * 256) to exp(0.6 * 256) in a segment of 256 slots."""
    t, c, n = 4096, 8, 4
    i = S.scan_inputs(1, t, c, n, F32, 31)
    i["a"] = torch.linspace(0.4, 0.6, c * n, device=L.DEV).reshape(c, n)
    i["dt_bias"] = torch.full((c,), math.log(math.e - 1.0), device=L.DEV)  # delta = 1
    i["dt"] *= 0.01
    i["x"][:, :t - 46] = 0.0
    i["dy"][:, 60:] = 0.0
    compare(call(L.positions(t, [[t]]), i), [[t]], i)


@pytest.mark.parametrize("t", [4096, 200])
def test_an_infinite_state_stays_infinite(t):
    """An infinite input, and an infinite gradient, are heard of for the rest of the sequence; whole segments' decays are 0 in 32 bits."""
    at, c, n = 100, 8, 8  # (as many states as a lane group holds)
    i = S.scan_inputs(1, t, c, n, F32, 32, z=False)
    for k in ("x", "b", "c", "dy", "d"):
        i[k] = i[k].abs() + 0.1
    i["a"] = -torch.linspace(1.0, 4.0, c * n, device=L.DEV).reshape(c, n)
    i["dt_bias"] = torch.full((c,), math.log(math.e - 1.0), device=L.DEV)
    pos = L.positions(t, [[t]])
    clean = call(pos, i)
    i["x"][0, at] = math.inf
    y = call(pos, i)["y"]
    i["x"][0, at] = 1.0
    i["dy"][0, t - at] = math.inf
    dx = call(pos, i)["dx"]
    torch.cuda.synchronize()
    assert torch.equal(y[0, :at], clean["y"][0, :at]) and torch.equal(dx[0, t - at + 1:], clean["dx"][0, t - at + 1:])
    assert bool((y[0, at:] == math.inf).all()) and bool((dx[0, :t - at + 1] == math.inf).all())
