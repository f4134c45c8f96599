"""bload_recurrence with infinities in a sequence: gates are above 0, so an infinite state stays infinite to the sequence's end, and an
infinite gradient to its start, however small the product of the gates between is."""
import math

import pytest
import torch

import layer_util as L
from test_gpu_recurrence import BF, F32, call

pytestmark = pytest.mark.gpu
DEV = L.DEV


@pytest.mark.parametrize("gate", [-1.0, -14.0, -60.0, -86.0, -87.0, -95.0])
@pytest.mark.parametrize("dtype", [F32, BF], ids=["fp32", "bf16"])
@pytest.mark.parametrize("t,c", [(300, 64), (3001, 17), (6000, 8)])
def test_an_infinite_state_stays(t, c, dtype, gate):
    """(With few channels the slots are walked in segments, which hand their states on.)"""
    lengths, at = [100, t - 140, 20, -20], 130
    s0, s1 = 100, t - 40
    pos = L.positions(t, [lengths])
    g = L.normal((1, t, c), dtype, 1, gate, 0.25)
    x, dh = L.normal((1, t, c), dtype, 2), L.normal((1, t, c), dtype, 3)
    clean = {n: y.clone() for n, y in call(pos, g, x, dh).items() if n in ("h", "dx")}
    x[0, at, 0], x[0, at, 1] = math.inf, -math.inf
    dh[0, s1 - 5, 2], dh[0, s1 - 5, 3] = math.inf, -math.inf
    got = call(pos, g, x, dh)
    torch.cuda.synchronize()
    assert bool((got["h"][0, at:s1, 0] == math.inf).all()) and bool((got["h"][0, at:s1, 1] == -math.inf).all())
    assert bool((got["dx"][0, s0:s1 - 4, 2] == math.inf).all()) and bool((got["dx"][0, s0:s1 - 4, 3] == -math.inf).all())
    for n, rows, ch in (("h", slice(s0, at), 0), ("h", slice(s1, t), 0), ("h", slice(0, t), 4), ("dx", slice(s1 - 4, t), 2), ("dx", slice(0, s0), 2)):
        assert torch.equal(got[n][0, rows, ch], clean[n][0, rows, ch]), (n, ch)


@pytest.mark.parametrize("gate", [-60.0, -70.0])
def test_gates_of_small_values_keep_their_bits(gate):
    """f of 1e-26 and 4e-31, with states so large that it shows."""
    t, c = 200, 32
    pos = L.positions(t, [[t]])
    g = L.normal((1, t, c), F32, 1, gate, 0.1)
    x = L.normal((1, t, c), F32, 2, std=1e-3)
    x[0, ::2] *= 1e36
    x[0, 1::2] = 0.0  # these slots' states are the one before, times f
    got = call(pos, g, x)["h"]
    torch.cuda.synchronize()
    val, tol = L.recurrence([[t]], g, x)
    L.close(got, val["h"], tol["h"], "h")
