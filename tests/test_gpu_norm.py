"""bload_norm and its gradient against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import layer_util as L
import state_space_util as S
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu
DEV = L.DEV
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


def inputs(b, t, c, dtype, seed=1, mean=0.5):
    return (L.normal((b, t, c), dtype, seed, mean, 2.0), L.normal((b, t, c), dtype, seed + 1), L.normal((c,), F32, seed + 2, 1.0, 0.2),
            L.normal((c,), F32, seed + 3))


def call(pos, x, dy, w, bias, eps=1e-5, stream=None, o=None):
    c = x.shape[-1]
    if o is None:
        o = {n: torch.full(x.shape, 7.0, dtype=x.dtype, device=DEV) for n in ("y", "dx")}
        o |= {n: torch.full((c,), 7.0, device=DEV) for n in ("dweight", "dbias")}
        o["stats"], o["work"] = B.bload_norm_buffers(pos, x)
    B.bload_norm(pos, x, o["y"], w, bias, o["stats"], eps=eps, stream=stream)
    B.bload_norm_grad(pos, x, o["stats"], dy, o["dx"], w, o["dweight"], o["dbias"], o["work"], stream=stream)
    return o


def compare(o, blocks, x, dy, w, bias, eps=1e-5):
    torch.cuda.synchronize()
    val, tol = S.norm(blocks, x, w, bias, eps, dy)
    for n in ("stats", "y", "dx", "dweight", "dbias"):
        L.close(o[n], val[n], tol[n], n)


CASES = [(F32, [[1]], 1, 16), (BF, [[1], [-1]], 1, 8), (FP, [[2, 3, 1], [6], [-6]], 6, 33), (BF, [[60, -4], [64]], 64, 256),
         (F32, [[7, 90], [40, -57]], 97, 257), (BF, [[33], [30, -3]], 33, 2048), (FP, [[33]], 33, 2049), (BF, [[50]], 50, 2056),
         (F32, [[20, -3]], 23, 5000), (FP, [[11, 2]], 13, 8192), (F32, [[9]], 9, 8193), (BF, [[9, -1]], 10, 16384), (F32, [[5]], 5, 16384),
         (BF, [[700, 301], [1, -1000]], 1001, 96), (FP, [[400]], 400, 1027)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%d" % (str(c[0])[6:], c[2], c[3]))
def test_values_and_gradients(case):
    dtype, blocks, t, c = case
    x, dy, w, bias = inputs(len(blocks), t, c, dtype)
    compare(call(L.positions(t, blocks), x, dy, w, bias), blocks, x, dy, w, bias)


@pytest.mark.parametrize("seed", range(6))
def test_random_packings(seed):
    rng = np.random.default_rng(seed)
    t, c, nb = int(rng.integers(1, 700)), int(rng.integers(3, 1500)), int(rng.integers(1, 5))
    blocks = L.random_blocks(rng, nb, t, 40.0)
    x, dy, w, bias = inputs(nb, t, c, [BF, FP, F32][seed % 3], 10 * seed)
    w, bias = (w if seed & 1 else None), (bias if seed & 2 else None)
    compare(call(L.positions(t, blocks), x, dy, w, bias), blocks, x, dy, w, bias)


def test_a_mean_far_from_zero_and_frames_without_spread():
    blocks, t, c = [[40, 24]], 64, 320
    x, dy, w, bias = inputs(1, t, c, F32, 3, mean=3000.0)
    x[0, 5] = 4.0  # all channels alike: 1 / sqrt(eps)
    x[0, 6, 0] = 1e6  # one outlier
    compare(call(L.positions(t, blocks), x, dy, w, bias), blocks, x, dy, w, bias)


@pytest.mark.parametrize("junk", [math.nan, math.inf])
def test_junk_on_padding_and_in_other_frames_stays_there(junk):
    blocks, t, c = [[50, -20, 30]], 100, 72
    x, dy, w, bias = inputs(1, t, c, BF)
    pos = L.positions(t, blocks)
    clean = call(pos, x, dy, w, bias)
    x[pos < 0], dy[pos < 0] = junk, junk
    got = call(pos, x, dy, w, bias)
    torch.cuda.synchronize()
    for n in ("stats", "y", "dx", "dweight", "dbias"):
        assert torch.equal(got[n], clean[n]), n
    assert all(bool((got[n][pos < 0] == 0).all()) for n in ("stats", "y", "dx"))
    x[0, 10] = junk
    got = call(pos, x, dy, w, bias)
    other = torch.arange(t, device=DEV) != 10
    assert torch.equal(got["y"][:, other], clean["y"][:, other]) and torch.equal(got["dx"][:, other], clean["dx"][:, other])
    assert not bool(torch.isfinite(got["y"][0, 10]).any())


def test_strides_and_broadcast_inputs():
    blocks, t, c = [[90, 60]] * 3, 150, 64
    pos = L.positions(t, blocks)
    x = L.normal((3, t, 2 * c), BF, 5)[..., c:]
    dy = L.normal((1, 1, c), BF, 6).expand(3, t, c)
    _, _, w, bias = inputs(3, t, c, BF)
    o = {"y": torch.full((t, 3, c), 7.0, dtype=BF, device=DEV).transpose(0, 1), "dx": torch.empty((3, t, c + 8), dtype=BF, device=DEV)[..., :c],
         "dweight": torch.empty(c, device=DEV), "dbias": torch.empty(c, device=DEV)}
    o["stats"], o["work"] = B.bload_norm_buffers(pos, x)
    compare(call(pos, x, dy, w, bias, o=o), blocks, x, dy, w, bias)
    odd = L.normal((3, t, c + 3), BF, 7)[..., 3:]  # rows that start on any element
    compare(call(pos, odd, dy, w, bias), blocks, odd, dy, w, bias)


def test_gradients_against_differences():
    blocks, t, c = [[40, 20, -4]], 64, 24
    x, dy, w, bias = inputs(1, t, c, F32, 3)
    o = call(L.positions(t, blocks), x, dy, w, bias)
    args = {"dx": x.double(), "dweight": w.double(), "dbias": bias.double()}
    for n in args:
        way = torch.randn(args[n].shape, dtype=torch.float64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
        ends = [float((S.norm(blocks, *[v + (e * way if k == n else 0) for k, v in args.items()], 1e-5)[0]["y"] * dy.double()).sum()) for e in (1e-4, -1e-4)]
        slope = (ends[0] - ends[1]) / 2e-4
        size = float((o[n].double() * way).abs().sum())
        assert abs(float((o[n].double() * way).sum()) - slope) <= 1e-5 * size, n


def test_repeated_calls_streams_and_graphs():
    rng = np.random.default_rng(2)
    blocks = L.random_blocks(rng, 3, 1500, 300.0)
    x, dy, w, bias = inputs(3, 1500, 200, BF)
    pos = L.positions(1500, blocks)
    want = call(pos, x, dy, w, bias)
    again = call(pos, x, dy, w, bias)

    def fresh():
        o = {n: torch.zeros_like(x) for n in ("y", "dx")} | {n: torch.zeros(200, device=DEV) for n in ("dweight", "dbias")}
        o["stats"], o["work"] = B.bload_norm_buffers(pos, x)
        return o

    s, o, r, g = torch.cuda.Stream(), fresh(), fresh(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    call(pos, x, dy, w, bias, stream=s, o=o)
    s.synchronize()
    with torch.cuda.graph(g):
        call(pos, x, dy, w, bias, o=r)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for n in ("stats", "y", "dx", "dweight", "dbias"):
        assert torch.equal(want[n], again[n]) and torch.equal(want[n], o[n]) and torch.equal(want[n], r[n]), n


def test_sums_that_are_not_wanted():
    blocks, t, c = [[30, 10]], 40, 48
    x, dy, w, bias = inputs(1, t, c, FP)
    pos = L.positions(t, blocks)
    want = call(pos, x, dy, w, bias)
    dx, db = torch.empty_like(x), torch.empty(c, device=DEV)
    B.bload_norm_grad(pos, x, want["stats"], dy, dx, w)
    torch.cuda.synchronize()
    assert torch.equal(dx, want["dx"])
    B.bload_norm_grad(pos, x, want["stats"], dy, dx, w, dbias=db, work=want["work"])
    y = torch.empty_like(x)
    B.bload_norm(pos, x, y, w, bias)
    torch.cuda.synchronize()
    assert torch.equal(db, want["dbias"]) and torch.equal(y, want["y"])


def test_rows_beyond_32_bits():
    c, far = 64, (1 << 31) + 64
    store = torch.empty(far + 64 * c, dtype=BF, device=DEV)
    x = torch.as_strided(store, (2, 50, c), (far, c, 1))
    x.copy_(L.normal((2, 50, c), BF, 3))
    blocks = [[50], [20, 30]]
    _, dy, w, bias = inputs(2, 50, c, BF)
    compare(call(L.positions(50, blocks), x, dy, w, bias), blocks, x, dy, w, bias)


def test_no_blocks_and_refusals():
    x = torch.empty((0, 64, 16), device=DEV)
    pos = torch.empty((0, 64), dtype=torch.int32, device=DEV)
    stats, work = B.bload_norm_buffers(pos, x)
    B.bload_norm(pos, x, torch.empty_like(x), None, None, stats)
    B.bload_norm_grad(pos, x, stats, x, torch.empty_like(x), None, torch.empty(16, device=DEV), None, work)
    x, dy, w, bias = inputs(2, 20, 16, F32)
    pos = L.positions(20, [[20], [10, 10]])
    y, (stats, work) = torch.empty_like(x), B.bload_norm_buffers(pos, x)
    for bad in (lambda: B.bload_norm(pos.float(), x, y), lambda: B.bload_norm(pos, x, y.half()), lambda: B.bload_norm(pos, x, y, w.half()),
                lambda: B.bload_norm(pos, x, y, w[:-1]), lambda: B.bload_norm(pos, x, y, w, bias, stats[:1]), lambda: B.bload_norm(pos, x.double(), y.double()),
                lambda: B.bload_norm(pos, x, y[:, :10]), lambda: B.bload_norm(pos, x, torch.empty((2, 16, 20), device=DEV).transpose(1, 2)),
                lambda: B.bload_norm_grad(pos, x, stats, dy, y, w, w.cpu())):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad, code in ((lambda: B.bload_norm(pos, x, y, eps=-1.0), -2), (lambda: B.bload_norm(pos, x, y[:, :1].expand(2, 20, 16)), -2),
                      (lambda: B.bload_norm_grad(pos, x, None, dy, y), -1), (lambda: B.bload_norm_grad(pos, x, stats, dy, y, w, w.clone()), -1),
                      (lambda: B.bload_norm_grad(pos, x, stats, dy, y, w, w.clone(), None, work[:16].clone()), -4)):
        with pytest.raises(B.BloadError) as e:
            bad()
        assert e.value.code == code
