"""bload_conv, its gradient and bload_conv_step against the definition in 64 bits."""
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


def inputs(b, t, c, taps, dtype, seed=1):
    return (L.normal((b, t, c), dtype, seed), L.normal((b, t, c), dtype, seed + 1), L.normal((c, taps), F32, seed + 2), L.normal((c,), F32, seed + 3))


def call(pos, x, dy, w, bias, act=True, stream=None, o=None):
    if o is None:
        o = {n: torch.full(x.shape, 7.0, dtype=x.dtype, device=DEV) for n in ("y", "dx")}
        o |= {"dweight": torch.full_like(w, 7.0), "dbias": torch.full((w.shape[0],), 7.0, device=DEV), "work": B.bload_conv_buffers(pos, x, w)}
    B.bload_conv(pos, x, o["y"], w, bias, silu=act, stream=stream)
    B.bload_conv_grad(pos, x, dy, o["dx"], w, o["dweight"], bias, o["dbias"], silu=act, work=o["work"], stream=stream)
    return o


def compare(o, blocks, x, dy, w, bias, act=True):
    torch.cuda.synchronize()
    val, tol, _ = S.conv(blocks, x, w, bias, act, dy)
    for n in ("y", "dx", "dweight", "dbias"):
        L.close(o[n], val[n], tol[n], n)


CASES = [(F32, [[1]], 1, 1, 4), (BF, [[1], [-1]], 1, 8, 2), (FP, [[2, 3, 1], [6], [-6]], 6, 5, 3), (BF, [[63], [62, -1]], 63, 64, 4),
         (F32, [[1] * 40, [2, 3] * 8], 40, 33, 4), (FP, [[31, 2, 1, 3, 32, 31]], 100, 128, 8), (BF, [[333], [-300, 33]], 333, 1032, 4),
         (F32, [[500]], 500, 250, 1), (BF, [[97, 3]], 100, 24, 7), (FP, [[700, 1, 2]], 703, 517, 2), (F32, [[90, -3, 7]], 100, 515, 5),
         (BF, [[3, -1, 2]], 6, 7, 8)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%d-%d" % (str(c[0])[6:], c[2], c[3], c[4]))
@pytest.mark.parametrize("act", [True, False])
def test_values_and_gradients(case, act):
    dtype, blocks, t, c, taps = case
    x, dy, w, bias = inputs(len(blocks), t, c, taps, dtype)
    compare(call(L.positions(t, blocks), x, dy, w, bias, act), blocks, x, dy, w, bias, act)


@pytest.mark.parametrize("seed", range(6))
def test_random_packings(seed):
    rng = np.random.default_rng(seed)
    t, c, nb = int(rng.integers(1, 1500)), int(rng.integers(1, 700)), int(rng.integers(1, 5))
    blocks = L.random_blocks(rng, nb, t, [2.0, 40.0, 300.0][seed % 3])
    x, dy, w, bias = inputs(nb, t, c, int(rng.integers(1, 9)), [BF, FP, F32][seed % 3], 10 * seed)
    bias = bias if seed & 1 else None
    compare(call(L.positions(t, blocks), x, dy, w, bias), blocks, x, dy, w, bias)


@pytest.mark.parametrize("junk", [math.nan, math.inf])
@pytest.mark.parametrize("taps", [4, 6])
def test_junk_on_padding_and_in_other_sequences_stays_there(junk, taps):
    blocks, t = [[50, 70, -30, 200, -50]], 400
    x, dy, w, bias = inputs(1, t, 48, taps, BF)
    pos = L.positions(t, blocks)
    clean = call(pos, x, dy, w, bias)
    bad = pos < 0
    x[bad], dy[bad] = junk, junk
    got = call(pos, x, dy, w, bias)
    torch.cuda.synchronize()
    for n in ("y", "dx", "dweight", "dbias"):
        assert torch.equal(got[n], clean[n]), n
    bad[0, 50:120] = True
    x[bad], dy[bad] = junk, junk
    got = call(pos, x, dy, w, bias)
    torch.cuda.synchronize()
    for n in ("y", "dx"):
        assert torch.equal(got[n][~bad], clean[n][~bad]), n
        assert bool((got[n][pos < 0] == 0).all()), n


def test_strides_and_broadcast_inputs():
    blocks, t, c = [[90, 60]] * 3, 150, 64
    pos = L.positions(t, blocks)
    _, _, w, bias = inputs(3, t, c, 4, BF)
    x = L.normal((3, t, 2 * c), BF, 5)[..., c:]
    dy = L.normal((1, 1, c), BF, 6).expand(3, t, c)
    o = {"y": torch.full((t, 3, c), 7.0, dtype=BF, device=DEV).transpose(0, 1), "dx": torch.empty((3, t, c + 8), dtype=BF, device=DEV)[..., :c],
         "dweight": torch.empty_like(w), "dbias": torch.empty(c, device=DEV), "work": B.bload_conv_buffers(pos, x, w)}
    compare(call(pos, x, dy, w, bias, o=o), blocks, x, dy, w, bias)
    odd = L.normal((3, t, c + 3), BF, 7)[..., 3:]
    compare(call(pos, odd, dy, w, bias), blocks, odd, dy, w, bias)


def test_gradients_against_differences():
    blocks, t, c = [[40, 20, -4]], 64, 6
    x, dy, w, bias = inputs(1, t, c, 4, F32, 3)
    o = call(L.positions(t, blocks), x, dy, w, bias)
    args = {"dx": x.double(), "dweight": w.double(), "dbias": bias.double()}
    for n in args:
        way = torch.randn(args[n].shape, dtype=torch.float64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
        ends = [float((S.conv(blocks, *[v + (e * way if k == n else 0) for k, v in args.items()], True)[0]["y"] * dy.double()).sum()) for e in (1e-4, -1e-4)]
        slope = (ends[0] - ends[1]) / 2e-4
        assert abs(float((o[n].double() * way).sum()) - slope) <= 1e-5 * float((o[n].double() * way).abs().sum()), n


def test_repeated_calls_streams_and_graphs():
    rng = np.random.default_rng(2)
    blocks = L.random_blocks(rng, 3, 1500, 300.0)
    x, dy, w, bias = inputs(3, 1500, 200, 4, BF)
    pos = L.positions(1500, blocks)
    want = call(pos, x, dy, w, bias)
    again = call(pos, x, dy, w, bias)

    def fresh():
        return {n: torch.zeros_like(x) for n in ("y", "dx")} | {"dweight": torch.zeros_like(w), "dbias": torch.zeros(200, device=DEV),
                                                                "work": B.bload_conv_buffers(pos, x, w)}

    s, o, r, g = torch.cuda.Stream(), fresh(), fresh(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    call(pos, x, dy, w, bias, stream=s, o=o)
    s.synchronize()
    with torch.cuda.graph(g):
        call(pos, x, dy, w, bias, o=r)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for n in ("y", "dx", "dweight", "dbias"):
        assert torch.equal(want[n], again[n]) and torch.equal(want[n], o[n]) and torch.equal(want[n], r[n]), n


def test_sums_that_are_not_wanted():
    blocks, t, c = [[30, 10]], 40, 48
    x, dy, w, bias = inputs(1, t, c, 4, FP)
    pos = L.positions(t, blocks)
    want = call(pos, x, dy, w, bias)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    B.bload_conv_grad(pos, x, dy, dx, w, bias=bias)
    torch.cuda.synchronize()
    assert torch.equal(dx, want["dx"])
    B.bload_conv_grad(pos, x, dy, dx, w, dw, bias=bias, work=want["work"])
    torch.cuda.synchronize()
    assert torch.equal(dw, want["dweight"])


def test_rows_beyond_32_bits():
    c, far = 64, (1 << 31) + 64
    store = torch.empty(far + 64 * c, dtype=BF, device=DEV)
    x = torch.as_strided(store, (2, 50, c), (far, c, 1))
    x.copy_(L.normal((2, 50, c), BF, 3))
    blocks = [[50], [20, 30]]
    _, dy, w, bias = inputs(2, 50, c, 4, BF)
    compare(call(L.positions(50, blocks), x, dy, w, bias), blocks, x, dy, w, bias)


@pytest.mark.parametrize("dtype,c,taps", [(BF, 64, 4), (F32, 7, 3), (FP, 130, 8), (BF, 24, 2), (F32, 515, 1)])
def test_tails_and_steps_go_on_where_a_packed_batch_ends(dtype, c, taps):
    blocks, t, more = [[1, 5, -2, 40], [-3, 2, 43]], 48, 3
    pos = L.positions(t, blocks)
    x, _, w, bias = inputs(2, t, c, taps, dtype)
    where = list(L.spans(blocks))
    n = len(where)
    ids, count = S.sequence_numbers(pos, torch.tensor([3, 0, 4, 1, 2], device=DEV))
    assert count == n
    tails = torch.full((n + 2, taps - 1, c), 5.0, dtype=dtype, device=DEV)  # two of other batches
    y = torch.empty_like(x)
    B.bload_conv(pos, x, y, w, bias, seq_id=ids, tails=tails if taps > 1 else None)
    torch.cuda.synchronize()
    assert bool((tails[n:] == 5.0).all())
    order = [3, 0, 4, 1, 2]
    val, tol, want = S.conv(blocks, x, w, bias, True)
    L.close(y, val["y"], tol["y"], "y")
    for k in range(n):
        assert torch.equal(tails[order[k]].double(), want[k]), k
    # three more frames of each, against the whole sequences
    state = tails[:n].clone()
    extra = L.normal((more, n, c), dtype, 9)
    whole = torch.zeros((n, t + more, c), dtype=dtype, device=DEV)
    lengths = []
    for k, (q, s0, s1) in enumerate(where):
        whole[order[k], :s1 - s0] = x[q, s0:s1]
        whole[order[k], s1 - s0:s1 - s0 + more] = extra[:, order[k]]
        lengths.append((order[k], s1 - s0))
    lengths = [m for _, m in sorted(lengths)]
    val, tol, _ = S.conv([[m + more] for m in lengths], whole, w, bias, True)
    for i in range(more):
        at = torch.tensor([m + i for m in lengths], dtype=torch.int32, device=DEV)
        out = torch.empty((n, c), dtype=dtype, device=DEV)
        B.bload_conv_step(at, state, extra[i].contiguous(), out, w, bias)
        torch.cuda.synchronize()
        rows = torch.arange(n, device=DEV)
        L.close(out, val["y"][rows, at.long()], tol["y"][rows, at.long()], "step %d" % i)


def test_steps_that_start_and_rows_without_a_frame():
    n, c, taps = 7, 36, 4
    w, bias = L.normal((c, taps), F32, 1), L.normal((c,), F32, 2)
    state, x = L.normal((n, taps - 1, c), BF, 3), L.normal((n, 2 * c), BF, 4)[:, c:]
    state[0], state[3], x[1], x[4] = math.nan, math.inf, math.nan, math.inf  # what starts or has no frame does not use them
    pos = torch.tensor([0, -1, 5, 0, -7, 1, 2], dtype=torch.int32, device=DEV)
    y, after, place = torch.empty((n, c), dtype=BF, device=DEV), torch.full_like(state, 7.0), state.clone()
    B.bload_conv_step(pos, state, x, y, w, bias, silu=False, next_state=after)
    y2 = torch.empty_like(y)
    B.bload_conv_step(pos, place, x, y2, w, bias, silu=False)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(after.nan_to_num(9.0), place.nan_to_num(9.0))
    for r, p in enumerate(pos.tolist()):
        if p < 0:
            assert bool((y[r] == 0).all()) and torch.equal(after[r], state[r])
            continue
        have = min(p, taps - 1)
        seen = torch.cat((S.zeros((taps - 1 - have, c)), state[r, taps - 1 - have:].double(), x[r:r + 1].double()))
        u = (seen * w.t().double()).sum(0) + bias.double()
        L.close(y[r], u, S.rounded(u, 6 * L.E * ((seen * w.t().double()).abs().sum(0) + bias.double().abs()), BF), "row %d" % r)
        assert torch.equal(after[r].double(), seen[1:])


def test_no_blocks_and_refusals():
    x = torch.empty((0, 64, 16), device=DEV)
    pos = torch.empty((0, 64), dtype=torch.int32, device=DEV)
    w = L.normal((16, 4), F32, 1)
    B.bload_conv(pos, x, torch.empty_like(x), w)
    B.bload_conv_grad(pos, x, x, torch.empty_like(x), w, torch.empty_like(w), work=B.bload_conv_buffers(pos, x, w))
    none = torch.empty(0, dtype=torch.int32, device=DEV)
    B.bload_conv_step(none, torch.empty((0, 3, 16), device=DEV), x[:, 0], x[:, 0].clone(), w)
    x, dy, w, bias = inputs(2, 20, 16, 4, F32)
    pos = L.positions(20, [[20], [10, 10]])
    y, work, ids = torch.empty_like(x), B.bload_conv_buffers(pos, x, w), S.sequence_numbers(pos)[0]
    at, state, row = pos[:, 0].contiguous(), torch.zeros((2, 3, 16), device=DEV), x[:, 0]
    for bad in (lambda: B.bload_conv(pos, x, y, w[:-1]), lambda: B.bload_conv(pos, x, y, w[0]), lambda: B.bload_conv(pos, x, y, w.half()),
                lambda: B.bload_conv(pos, x, y, w, tails=state), lambda: B.bload_conv(pos, x, y, w, seq_id=ids, tails=state[:, :2]),
                lambda: B.bload_conv(pos, x, y, w, seq_id=ids.long(), tails=state), lambda: B.bload_conv(pos, x, y[:, :3], w),
                lambda: B.bload_conv_grad(pos, x, dy, y, w, dweight=w[:, :3].clone()), lambda: B.bload_conv_step(at.long(), state, row, row.clone(), w),
                lambda: B.bload_conv_step(at, state[:, :2], row, row.clone(), w), lambda: B.bload_conv_step(at, state.half(), row, row.clone(), w),
                lambda: B.bload_conv_step(at[:1], state, row, row.clone(), w)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    wide = L.normal((16, 9), F32, 1)
    for bad, code in ((lambda: B.bload_conv(pos, x, y, wide), -6), (lambda: B.bload_conv(pos, x, y[:, :1].expand(2, 20, 16), w), -2),
                      (lambda: B.bload_conv_grad(pos, x, dy, y, w, w.clone()), -1),
                      (lambda: B.bload_conv_grad(pos, x, dy, y, w, w.clone(), work=work[:64].clone()), -4)):
        with pytest.raises(B.BloadError) as e:
            bad()
        assert e.value.code == code
