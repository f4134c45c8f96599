"""bload_recurrence and its gradient against the definition in 64 bits, one sequence at a time."""
import math

import numpy as np
import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu
DEV = L.DEV
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


def call(pos, gate, x, dh=None, stream=None, o=None):
    o = {n: torch.full(x.shape, 7.0, dtype=x.dtype, device=DEV) for n in ("h", "dgate", "dx")} if o is None else o
    o["carry"], o["work"] = B.bload_recurrence_buffers(pos, x) if "carry" not in o else (o["carry"], o["work"])
    B.bload_recurrence(pos, gate, x, o["h"], o["carry"], o["work"], stream=stream)
    if dh is not None:
        B.bload_recurrence_grad(pos, gate, x, o["carry"], dh, o["dgate"], o["dx"], o["work"], stream=stream)
    return o


def inputs(b, t, c, dtype, seed=1, mean=2.0):
    return L.normal((b, t, c), dtype, seed, mean, 1.5), L.normal((b, t, c), dtype, seed + 1), L.normal((b, t, c), dtype, seed + 2)


def compare(o, blocks, gate, x, dh=None):
    torch.cuda.synchronize()
    val, tol = L.recurrence(blocks, gate, x, dh)
    for n in ("h",) if dh is None else ("h", "dgate", "dx"):
        L.close(o[n], val[n], tol[n], n)


CASES = [
    (F32, [[1]], 1, 1), (BF, [[1], [-1]], 1, 8), (FP, [[2, 3, 1], [6], [-6]], 6, 5), (BF, [[63], [62, -1]], 63, 64),
    (F32, [[64], [63, 1], [1, 63]], 64, 128), (BF, [[65], [64, 1], [1, 64]], 65, 136), (FP, [[128], [64, 64]], 128, 256),
    (F32, [[129], [60, 60, -9]], 129, 33), (BF, [[500], [100, 300, 100], [1] * 500], 500, 72),
    (BF, [[2000], [-1000, 1000], [130, 700, -170, 1000]], 2000, 40), (F32, [[3001]], 3001, 17), (F32, [[3001]], 3001, 256),
    (FP, [[1000], [3, 500, 497]], 1000, 1000), (BF, [[300, 5]], 305, 1), (BF, [[300, 5]], 305, 2051),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%d" % (str(c[0])[6:], c[2], c[3]))
def test_values_and_gradients(case):
    dtype, blocks, t, c = case
    gate, x, dh = inputs(len(blocks), t, c, dtype)
    compare(call(L.positions(t, blocks), gate, x, dh), blocks, gate, x, dh)


@pytest.mark.parametrize("seed", range(6))
def test_random_packings(seed):
    rng = np.random.default_rng(seed)
    t, c, nb = int(rng.integers(1, 1500)), int(rng.integers(1, 400)), int(rng.integers(1, 5))
    blocks = L.random_blocks(rng, nb, t, [3.0, 40.0, 300.0][seed % 3])
    gate, x, dh = inputs(nb, t, c, [BF, FP, F32][seed % 3], 50 * seed)
    compare(call(L.positions(t, blocks), gate, x, dh), blocks, gate, x, dh)


@pytest.mark.parametrize("mean", [-8.0, 0.0, 8.0])
def test_gates_far_open_and_far_closed(mean):
    blocks = [[700, 200, -100]]
    gate, x, dh = inputs(1, 1000, 24, F32, 9, mean)
    gate[0, ::50] = 100.0   # f = 1: carries on for ever
    gate[0, 7::50] = -100.0  # f = 0: forgets all
    compare(call(L.positions(1000, blocks), gate, x, dh), blocks, gate, x, dh)


def test_longest_block():
    blocks = [[30000, 2768]]
    gate, x, dh = inputs(1, 32768, 9, F32, 4)
    compare(call(L.positions(32768, blocks), gate, x, dh), blocks, gate, x, dh)


def test_many_blocks():
    nb = 70000  # more than a grid's second dimension holds
    pos = torch.tensor([[0, 1, -1]], dtype=torch.int32, device=DEV).repeat(nb, 1)
    gate, x, dh = inputs(nb, 3, 2, F32)
    o = call(pos, gate, x, dh)
    f = torch.sigmoid(gate.double())
    h0 = (1 - f[:, 0]) * x[:, 0].double()
    h1 = f[:, 1] * h0 + (1 - f[:, 1]) * x[:, 1].double()
    g0 = dh[:, 0].double() + f[:, 1] * dh[:, 1].double()
    assert torch.allclose(o["h"][:, 0].double(), h0, atol=1e-5) and torch.allclose(o["h"][:, 1].double(), h1, atol=1e-5)
    assert torch.allclose(o["dx"][:, 0].double(), (1 - f[:, 0]) * g0, atol=1e-5)
    assert bool((o["h"][:, 2] == 0).all()) and bool((o["dx"][:, 2] == 0).all()) and bool((o["dgate"][:, 2] == 0).all())


@pytest.mark.parametrize("junk", [math.nan, math.inf])
def test_junk_on_padding_and_in_other_sequences_stays_there(junk):
    blocks, t = [[50, 70, -30, 200, -50]], 400
    gate, x, dh = inputs(1, t, 48, BF)
    pos = L.positions(t, blocks)
    clean = call(pos, gate, x, dh)
    bad = torch.zeros((1, t), dtype=torch.bool, device=DEV)
    bad[0, 50:150] = True
    bad[0, 350:] = True
    for y in (gate, x, dh):
        y[bad] = junk
    got = call(pos, gate, x, dh)
    torch.cuda.synchronize()
    for n in ("h", "dgate", "dx"):
        assert torch.equal(got[n][~bad], clean[n][~bad]), n
        assert bool((got[n][pos < 0] == 0).all()), n


def test_strides_and_broadcast_inputs():
    blocks, t, c = [[90, 60]] * 3, 150, 64
    pos = L.positions(t, blocks)
    both = L.normal((3, t, 2 * c), BF, 5)
    gate, x = both[..., :c], both[..., c:]
    dh = L.normal((1, 1, c), BF, 6).expand(3, t, c)
    grads = torch.full((3, t, 2 * c), 5.0, dtype=BF, device=DEV)
    o = {"h": torch.full((t, 3, c), 7.0, dtype=BF, device=DEV).transpose(0, 1), "dgate": grads[..., :c], "dx": grads[..., c:]}
    compare(call(pos, gate, x, dh, o=o), blocks, gate, x, dh)
    odd = L.normal((3, t, c + 3), BF, 7)[..., 3:]  # rows that start on any element
    compare(call(pos, gate, odd, dh), blocks, gate, odd, dh)


def test_gradients_against_differences():
    blocks, t, c = [[40, 20, -4]], 64, 6
    gate, x, dh = inputs(1, t, c, F32, 3, 0.5)
    o = call(L.positions(t, blocks), gate, x, dh)
    _, tol = L.recurrence(blocks, gate, x, dh)
    base = [gate.double(), x.double()]
    for n, name in enumerate(("dgate", "dx")):
        way = torch.randn(x.shape, dtype=torch.float64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(n))
        ends = []
        for e in (1e-4, -1e-4):
            args = list(base)
            args[n] = args[n] + e * way
            ends.append(float((L.recurrence(blocks, *args)[0]["h"] * dh.double()).sum()))
        slope = (ends[0] - ends[1]) / 2e-4
        assert abs(float((o[name].double() * way).sum()) - slope) <= float((tol[name] * way.abs()).sum()) + 1e-6 * abs(slope) + 1e-7, name


def test_repeated_calls_streams_and_graphs():
    rng = np.random.default_rng(2)
    blocks = L.random_blocks(rng, 3, 2500, 700.0)
    gate, x, dh = inputs(3, 2500, 200, BF)
    pos = L.positions(2500, blocks)
    want = {n: y.clone() for n, y in call(pos, gate, x, dh).items() if n in ("h", "dgate", "dx", "carry")}
    again = call(pos, gate, x, dh)
    s = torch.cuda.Stream()
    o = {n: torch.empty_like(x) for n in ("h", "dgate", "dx")}
    o["carry"], o["work"] = B.bload_recurrence_buffers(pos, x)
    s.wait_stream(torch.cuda.current_stream())
    call(pos, gate, x, dh, stream=s, o=o)
    s.synchronize()
    g, r = torch.cuda.CUDAGraph(), {n: torch.empty_like(x) for n in ("h", "dgate", "dx")}
    r["carry"], r["work"] = B.bload_recurrence_buffers(pos, x)
    with torch.cuda.graph(g):
        call(pos, gate, x, dh, o=r)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for n in want:
        assert torch.equal(want[n], again[n]) and torch.equal(want[n], o[n]) and torch.equal(want[n], r[n]), n


def test_without_carry():
    blocks = [[100, 29], [129]]
    gate, x, _ = inputs(2, 129, 40, FP)
    pos = L.positions(129, blocks)
    want = call(pos, gate, x)["h"]
    h = torch.empty_like(x)
    B.bload_recurrence(pos, gate, x, h, None, B.bload_recurrence_buffers(pos, x)[1])
    torch.cuda.synchronize()
    assert torch.equal(h, want)


def test_no_blocks():
    x = torch.empty((0, 64, 16), device=DEV)
    pos = torch.empty((0, 64), dtype=torch.int32, device=DEV)
    carry, work = B.bload_recurrence_buffers(pos, x)
    B.bload_recurrence(pos, x, x, torch.empty_like(x), carry, work)
    B.bload_recurrence_grad(pos, x, x, carry, x, torch.empty_like(x), torch.empty_like(x), work)
    torch.cuda.synchronize()


def test_refusals():
    gate, x, dh = inputs(2, 200, 16, F32)
    pos = L.positions(200, [[200], [100, 100]])
    h, (carry, work) = torch.empty_like(x), B.bload_recurrence_buffers(pos, x)
    with pytest.raises(TypeError):
        B.bload_recurrence(pos.short(), gate, x, h, carry, work)
    with pytest.raises(TypeError):
        B.bload_recurrence(pos, gate.double(), x, h, carry, work)
    with pytest.raises(TypeError):
        B.bload_recurrence(pos, gate.double(), x.double(), h.double(), carry, work)
    with pytest.raises(TypeError):
        B.bload_recurrence(pos, gate, x, h, carry[:, :1], work)
    with pytest.raises(ValueError):
        B.bload_recurrence(pos, gate[:, :100], x, h, carry, work)
    with pytest.raises(ValueError):
        B.bload_recurrence(pos, gate, x, torch.empty((2, 16, 200), device=DEV).transpose(1, 2), carry, work)
    for bad, code in ((h[:, :1].expand(2, 200, 16), -2),):
        with pytest.raises(B.BloadError) as e:
            B.bload_recurrence(pos, gate, x, bad, carry, work)
        assert e.value.code == code
    with pytest.raises(B.BloadError) as e:
        B.bload_recurrence_grad(pos, gate, x, None, dh, h, torch.empty_like(x), work)
    assert e.value.code == -1
