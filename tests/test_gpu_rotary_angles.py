"""Sine and cosine of bload_rotary's angles, by themselves: pairs (1, 0) in 32 bits come out as (cos a, sin a).

Bound: the angle is reduced to |r| <= 0.8 with an error of two roundings of r (2 * 2^-25), the series leave 3e-8 and round their last
three steps (3 * 2^-25); sincosf is within two units in the last place.  Both are within 4 * 2^-24."""
import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu
DEV = L.DEV


@pytest.mark.parametrize("span", [(0.001, 1.0), (1.0, 20.0), (20.0, 120.0), (120.0, 1000.0), (1000.0, 1e5)],
                         ids=lambda s: "%g" % s[1])
def test_sine_and_cosine(span):
    t, n = 8192, 256
    pos = L.positions(t, [[t]])
    inv = torch.empty(n, dtype=torch.float64).uniform_(*span, generator=torch.Generator().manual_seed(3)).float().to(DEV)
    x = torch.zeros((1, t, 1, 2 * n), device=DEV)
    x[..., :n] = 1.0
    y = torch.empty_like(x)
    B.bload_rotary(pos, x, y, inv)
    torch.cuda.synchronize()
    a = (pos[..., None].float() * inv).double()[:, :, None]
    want = torch.cat((a.cos(), a.sin()), -1)
    L.close(y, want, torch.full_like(want, 4 * 2.0 ** -24), "cos, sin")
