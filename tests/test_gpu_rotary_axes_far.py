"""Sine and cosine of bload_rotary_axes at the far end of the range that it reduces by itself, read off a turned unit vector."""
import numpy as np
import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu

# Of an angle a + rest below 3e5, where rest is what the product's rounding left out of a: the reduced angle r is at most 0.82, and errs by
# a rounding each of two multiply-adds and one addition (2^-25 below 1).  Series remainders are at most 4e-8; the series' own
# arithmetic takes two roundings of at most 2^-24, and the element's multiply-add one.
TOL = 3 * 2.0 ** -25 + 4e-8 + 3 * 2.0 ** -24


@pytest.mark.parametrize("lo,hi", [(2.0 ** 18, 3e5), (2.0 ** 17, 2.0 ** 18), (100.0, 2.0 ** 17), (3e5, 3.1e5)])
@pytest.mark.parametrize("grad", [False, True])
def test_sine_and_cosine_of_products_that_need_rounding(lo, hi, grad):
    rng = np.random.default_rng(5)
    t, n = 4096, 64
    pos = L.positions(t, [[t]])
    near = 2 * lo >= hi  # then frequencies near 1, so that all angles are in the range; otherwise from 0.5 on
    inv = 1.0 - rng.uniform(0.0, 0.5, n) * (2.0 ** -8 if near else 1.0)
    inv = torch.from_numpy(inv.astype(np.float32)).to(L.DEV)
    coords = torch.from_numpy(rng.integers(int(lo if near else 2 * lo), int(hi), (1, 1, t), dtype=np.int32)).to(L.DEV)
    axis = torch.zeros(n, dtype=torch.int32, device=L.DEV)
    x = torch.zeros((1, t, 1, 2 * n), device=L.DEV)
    x[..., :n] = 1.0
    y = torch.empty_like(x)
    (B.bload_rotary_axes_grad if grad else B.bload_rotary_axes)(pos, coords, axis, x, y, inv)
    torch.cuda.synchronize()
    a = coords[0, 0].double()[:, None] * inv.double()
    want = torch.cat((a.cos(), -a.sin() if grad else a.sin()), -1)[None, :, None]
    L.close(y, want, torch.full_like(want, TOL), "turned")
