"""bload_rotary and its gradient against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu
DEV = L.DEV
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


def freq(rot, base=10000.0):
    return (base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / max(rot, 1))).float().to(DEV)


def reference(pos, x, inv, interleaved, factor, grad):
    """(value, allowed error).  The angle is the product rounded to 32 bits, so its sine and cosine are taken of that; they
    and their products with the elements are then off by a few roundings (8 of them allowed: argument reduction of an
    angle up to 32,768 turns included), and the result is rounded once."""
    n = inv.numel()
    a = (pos[..., None].float() * inv).double()[:, :, None]
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


def check(pos, x, inv, interleaved=False, factor=1.0, y=None, stream=None):
    for grad, fn in ((False, B.bload_rotary), (True, B.bload_rotary_grad)):
        want, tol = reference(pos, x, inv, interleaved, factor, grad)
        out = torch.full(x.shape, 7.0, dtype=x.dtype, device=DEV) if y is None else y
        fn(pos, x, out, inv, interleaved=interleaved, factor=factor, stream=stream)
        torch.cuda.synchronize()
        L.close(out, want, tol, "grad" if grad else "value")


CASES = [
    (F32, [[1]], 1, 1, 2, 2, False, 1.0), (BF, [[1], [-1]], 1, 1, 8, 8, True, 1.0), (FP, [[2, 4], [6]], 6, 3, 64, 64, False, 1.0),
    (BF, [[30, 34], [60, -4]], 64, 16, 64, 64, False, 1.0), (BF, [[30, 34], [60, -4]], 64, 5, 128, 64, True, 1.0),
    (F32, [[100, 1], [101]], 101, 4, 80, 32, True, 1.2), (FP, [[100, 1], [101]], 101, 4, 80, 32, False, 1.2),
    (BF, [[333]], 333, 2, 96, 40, False, 1.0), (BF, [[333]], 333, 3, 24, 18, True, 0.5), (F32, [[333]], 333, 3, 7, 6, False, 1.0),
    (FP, [[333]], 333, 33, 17, 0, False, 1.0), (BF, [[333]], 333, 1, 13, 12, True, 2.0), (F32, [[50, -20]], 70, 40, 128, 128, True, 1.0),
    (BF, [[4096]], 4096, 2, 128, 128, False, 1.0), (F32, [[32768]], 32768, 1, 64, 64, False, 1.0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%dx%d-%d%s" % (str(c[0])[6:], c[2], c[3], c[4], c[5], "i" if c[6] else ""))
def test_values_and_gradients(case):
    dtype, blocks, t, h, d, rot, interleaved, factor = case
    x = L.normal((len(blocks), t, h, d), dtype, 3)
    check(L.positions(t, blocks), x, freq(rot), interleaved, factor)


@pytest.mark.parametrize("seed", range(6))
def test_random_packings(seed):
    rng = np.random.default_rng(seed)
    t, h, d, nb = int(rng.integers(1, 700)), int(rng.integers(1, 12)), int(rng.integers(1, 140)), int(rng.integers(1, 4))
    x = L.normal((nb, t, h, d), [F32, FP, BF][seed % 3], seed)
    pos = L.positions(t, L.random_blocks(rng, nb, t, 50.0))
    check(pos, x, freq(2 * int(rng.integers(0, d // 2 + 1))), bool(seed & 1), 1.0 + 0.1 * seed)


def test_any_frequencies():
    pos = L.positions(3000, [[3000]])
    x = L.normal((1, 3000, 2, 16), F32, 3)
    check(pos, x, torch.tensor([1000.0, 50.0, 6.2831855, 3.1415927, 1.0, 0.0, -2.5, 1e-9], device=DEV))
    check(pos, x, torch.tensor([1e6, 123456.7, -4e5], device=DEV), True)


def test_in_place_strides_and_streams():
    blocks, t = [[50, 70, -10]] * 2, 130
    pos = L.positions(t, blocks)
    qkv = L.normal((2, t, 12, 64), BF, 2)
    x = qkv[:, :, :8]
    inv = freq(64)
    want, tol = reference(pos, x, inv, False, 1.0, False)
    rest = qkv[:, :, 8:].clone()
    B.bload_rotary(pos, x, x, inv)
    torch.cuda.synchronize()
    L.close(x, want, tol, "in place")
    assert torch.equal(qkv[:, :, 8:], rest)
    part = L.normal((2, t, 6, 40), BF, 2)  # copied elements in place, too
    want, tol = reference(pos, part, freq(16), True, 1.0, False)
    B.bload_rotary(pos, part, part, freq(16), interleaved=True)
    torch.cuda.synchronize()
    L.close(part, want, tol, "in place, partial")
    hf = L.normal((2, 6, t, 64), FP, 3).transpose(1, 2)
    check(pos, hf, inv, y=torch.empty((2, 6, t, 64), dtype=FP, device=DEV).transpose(1, 2))
    odd = L.normal((2, t, 5, 67), BF, 4)[..., 3:]
    check(pos, odd, inv)
    check(pos, L.normal((1, 1, 1, 64), F32, 5).expand(2, t, 3, 64), inv)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check(pos, hf, inv, stream=s)


def test_the_gradient_undoes_the_turn_and_agrees_with_differences():
    blocks, t = [[40, 24]], 64
    pos, inv = L.positions(t, blocks), freq(32)
    x, dy = L.normal((1, t, 2, 32), F32, 1), L.normal((1, t, 2, 32), F32, 2)
    y, back, dx, moved = (torch.empty_like(x) for _ in range(4))
    B.bload_rotary(pos, x, y, inv)
    B.bload_rotary_grad(pos, y, back, inv)
    B.bload_rotary_grad(pos, dy, dx, inv, factor=1.3)
    way = L.normal(x.shape, F32, 3)
    B.bload_rotary(pos, way, moved, inv, factor=1.3)  # linear in x: the difference quotient is the map itself
    torch.cuda.synchronize()
    assert float((back - x).abs().max()) <= 32 * L.E * float(x.abs().max()) * 2
    a, b = float((dx.double() * way.double()).sum()), float((dy.double() * moved.double()).sum())
    assert abs(a - b) <= 32 * L.E * float((dx.double() * way.double()).abs().sum())


def test_no_blocks_and_refusals():
    x = torch.empty((0, 64, 2, 64), dtype=BF, device=DEV)
    B.bload_rotary(torch.empty((0, 64), dtype=torch.int32, device=DEV), x, torch.empty_like(x), freq(64))
    pos = L.positions(64, [[64]])
    x = L.normal((1, 64, 2, 64), BF, 1)
    y, inv = torch.empty_like(x), freq(64)
    with pytest.raises(TypeError):
        B.bload_rotary(pos.float(), x, y, inv)
    with pytest.raises(TypeError):
        B.bload_rotary(pos, x, y.float(), inv)
    with pytest.raises(TypeError):
        B.bload_rotary(pos, x, y, inv.double())
    with pytest.raises(ValueError):
        B.bload_rotary(pos, x, y[:, :, :1], inv)
    with pytest.raises(TypeError):
        B.bload_rotary(pos, x.double(), y.double(), inv)
    for bad, code in ((lambda: B.bload_rotary(pos, x, y, freq(66)), -2),
                      (lambda: B.bload_rotary(pos, x, y[:, :1].expand(1, 64, 2, 64), inv), -2),
                      (lambda: B.bload_rotary(pos, x, y, inv, factor=float("inf")), -2)):
        with pytest.raises(B.BloadError) as e:
            bad()
        assert e.value.code == code
