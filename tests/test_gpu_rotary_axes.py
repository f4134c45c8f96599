"""bload_rotary_axes and its gradient against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu
DEV = L.DEV
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


def reference(pos, coords, axis, x, inv, interleaved, factor, grad):
    """(value, allowed error): the angle is the exact product, sine and cosine of it and the products with the elements are off by a few
    roundings (8 of them), and the result is rounded once."""
    n = inv.numel()
    known = (axis >= 0) & (axis < coords.shape[0])
    at = coords.permute(1, 2, 0)[..., axis.long().clamp(0, coords.shape[0] - 1)].float().double() * known
    a = (at * inv.double())[:, :, None]
    c, s = factor * a.cos(), factor * a.sin() * (-1 if grad else 1)
    X = x.double()
    y, tol = X.clone(), torch.zeros_like(X)
    iu = slice(0, 2 * n, 2) if interleaved else slice(0, n)
    iw = slice(1, 2 * n, 2) if interleaved else slice(n, 2 * n)
    u, w = X[..., iu], X[..., iw]
    y[..., iu], y[..., iw] = u * c - w * s, w * c + u * s
    slack = 8 * L.E * abs(factor) * (u.abs() + w.abs())
    tol[..., iu], tol[..., iw] = slack, slack
    tol[..., :2 * n] += L.U[x.dtype] * y[..., :2 * n].abs() + (2.0 ** -25 if x.dtype == FP else 0.0)
    pad = pos < 0
    y[pad], tol[pad] = X[pad], 0.0
    return y, tol


def check(pos, coords, axis, x, inv, interleaved=False, factor=1.0, y=None, stream=None):
    for grad, fn in ((False, B.bload_rotary_axes), (True, B.bload_rotary_axes_grad)):
        want, tol = reference(pos, coords, axis, x, inv, interleaved, factor, grad)
        out = torch.full(x.shape, 7.0, dtype=x.dtype, device=DEV) if y is None else y
        fn(pos, coords, axis, x, out, inv, interleaved=interleaved, factor=factor, stream=stream)
        torch.cuda.synchronize()
        L.close(out, want, tol, "grad" if grad else "value")


def inputs(rng, pos, axes, n, far=5000):
    """coordinates, the axis and the frequency of each pair"""
    coords = torch.from_numpy(rng.integers(-20, far, (axes, *pos.shape)).astype(np.int32)).to(DEV)
    return coords, torch.from_numpy(rng.integers(0, axes, n).astype(np.int32)).to(DEV), (10000.0 ** (-torch.arange(n) / max(n, 1))).float().to(DEV)


CASES = [(F32, [[1]], 1, 1, 2, 2, 3, False, 1.0), (BF, [[1], [-1]], 1, 1, 8, 8, 2, True, 1.0), (FP, [[2, 4], [6]], 6, 3, 64, 64, 1, False, 1.0),
         (BF, [[30, 34], [60, -4]], 64, 16, 64, 64, 3, False, 1.0), (BF, [[30, 34], [60, -4]], 64, 5, 128, 64, 4, True, 1.0),
         (F32, [[100, 1], [101]], 101, 4, 80, 32, 3, True, 1.2), (FP, [[100, 1], [101]], 101, 4, 80, 32, 3, False, 1.2),
         (BF, [[333]], 333, 3, 24, 18, 2, True, 0.5), (F32, [[333]], 333, 3, 7, 6, 3, False, 1.0), (FP, [[333]], 333, 33, 17, 0, 3, False, 1.0),
         (BF, [[333]], 333, 1, 13, 12, 3, True, 2.0), (BF, [[2000]], 2000, 20, 128, 128, 3, False, 1.0)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%dx%d-%d-%d%s" % (str(c[0])[6:], c[2], c[3], c[4], c[5], c[6], "i" if c[7] else ""))
def test_values_and_gradients(case):
    dtype, blocks, t, h, d, rot, axes, interleaved, factor = case
    pos = L.positions(t, blocks)
    check(pos, *inputs(np.random.default_rng(1), pos, axes, rot // 2)[:2], L.normal((len(blocks), t, h, d), dtype, 3),
          inputs(np.random.default_rng(1), pos, axes, rot // 2)[2], interleaved, factor)


@pytest.mark.parametrize("interleaved", [False, True])
def test_sections_of_axes_and_far_coordinates(interleaved):
    t = 600
    pos = L.positions(t, [[t]])
    x = L.normal((1, t, 5, 128), F32, 3)
    p = torch.arange(t, device=DEV, dtype=torch.int32)[None]
    for base in (0, 30000, 1 << 23):  # angles of whole radians: with the product rounded the last would be off by half a radian
        coords = torch.stack((p + base, p // 32 % 18, -(p % 32)))
        i = torch.arange(64, device=DEV)
        axis = torch.where(i < 16, 0, torch.where(i < 40, 1, 2)).to(torch.int32)
        check(pos, coords, axis, x, (10000.0 ** (-i.double() / 64)).float(), interleaved)
    check(pos, coords, axis, x, torch.full((64,), 777.7, device=DEV), interleaved)  # angles of 6e9


def test_one_axis_is_the_plain_rotary():
    blocks, t = [[50, 70, -10]] * 2, 130
    pos = L.positions(t, blocks)
    x = L.normal((2, t, 4, 64), BF, 2)
    inv = torch.tensor([2.0 ** -i for i in range(32)], device=DEV)  # products that need no rounding
    y, z = torch.empty_like(x), torch.empty_like(x)
    B.bload_rotary(pos, x, y, inv)
    B.bload_rotary_axes(pos, pos[None].contiguous(), torch.zeros(32, dtype=torch.int32, device=DEV), x, z, inv)
    torch.cuda.synchronize()
    assert torch.equal(y, z)


def test_in_place_strides_streams_and_graphs():
    blocks, t = [[50, 70, -10]] * 2, 130
    pos = L.positions(t, blocks)
    coords, axis, inv = inputs(np.random.default_rng(2), pos, 3, 32)
    qkv = L.normal((2, t, 12, 64), BF, 2)
    x, rest = qkv[:, :, :8], qkv[:, :, 8:].clone()
    want, tol = reference(pos, coords, axis, x, inv, False, 1.0, False)
    B.bload_rotary_axes(pos, coords, axis, x, x, inv)
    torch.cuda.synchronize()
    L.close(x, want, tol, "in place")
    assert torch.equal(qkv[:, :, 8:], rest)
    hf = L.normal((2, 6, t, 64), FP, 3).transpose(1, 2)
    check(pos, coords, axis, hf, inv, y=torch.empty((2, 6, t, 64), dtype=FP, device=DEV).transpose(1, 2))
    check(pos, coords, axis, L.normal((2, t, 5, 67), BF, 4)[..., 3:], inv)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check(pos, coords, axis, hf, inv, stream=s)
    once, again, g = torch.empty_like(hf), torch.empty_like(hf), torch.cuda.CUDAGraph()
    B.bload_rotary_axes(pos, coords, axis, hf, once, inv)
    with torch.cuda.graph(g):
        B.bload_rotary_axes(pos, coords, axis, hf, again, inv)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(once, again)


def test_an_axis_that_there_is_not_counts_as_coordinate_zero():
    pos = L.positions(40, [[40]])
    coords, _, inv = inputs(np.random.default_rng(3), pos, 2, 8)
    axis = torch.tensor([0, 1, 2, -1, 1 << 30, -(1 << 31), 1, 0], dtype=torch.int32, device=DEV)
    check(pos, coords, axis, L.normal((1, 40, 3, 16), F32, 1), inv, factor=1.5)


def test_no_blocks_and_refusals():
    x = torch.empty((0, 64, 2, 64), dtype=BF, device=DEV)
    pos = torch.empty((0, 64), dtype=torch.int32, device=DEV)
    inv, axis = torch.ones(32, device=DEV), torch.zeros(32, dtype=torch.int32, device=DEV)
    B.bload_rotary_axes(pos, torch.empty((3, 0, 64), dtype=torch.int32, device=DEV), axis, x, torch.empty_like(x), inv)
    pos = L.positions(64, [[64]])
    x, coords = L.normal((1, 64, 2, 64), BF, 1), torch.zeros((3, 1, 64), dtype=torch.int32, device=DEV)
    y = torch.empty_like(x)
    for bad in (lambda: B.bload_rotary_axes(pos, coords.long(), axis, x, y, inv), lambda: B.bload_rotary_axes(pos, coords[:, :, :60], axis, x, y, inv),
                lambda: B.bload_rotary_axes(pos, coords, axis[:5], x, y, inv), lambda: B.bload_rotary_axes(pos, coords, axis.long(), x, y, inv),
                lambda: B.bload_rotary_axes(pos, coords.cpu(), axis, x, y, inv), lambda: B.bload_rotary_axes(pos, coords[0], axis, x, y, inv)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad, code in ((lambda: B.bload_rotary_axes(pos, coords[:1].expand(5, 1, 64).contiguous(), axis, x, y, inv), -2),
                      (lambda: B.bload_rotary_axes(pos, coords[:0], axis, x, y, inv), -2),
                      (lambda: B.bload_rotary_axes(pos, coords, axis, x, y, inv, factor=float("inf")), -2)):
        with pytest.raises(B.BloadError) as e:
            bad()
        assert e.value.code == code
