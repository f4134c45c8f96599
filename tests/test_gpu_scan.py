"""bload_scan, its gradient and bload_scan_step against the definition in 64 bits, one sequence at a time."""
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
FRAMES, SUMS = ("y", "dx", "ddt", "dz"), ("db", "dc", "da", "dd", "ddt_bias")


def fresh(pos, i):
    o = {n: torch.full(i["x"].shape, 7.0, dtype=i["x"].dtype, device=DEV) for n in FRAMES}
    o |= {"db": torch.full(i["b"].shape, 7.0, dtype=i["x"].dtype, device=DEV), "da": torch.full_like(i["a"], 7.0)}
    o["dc"] = o["db"].clone()
    o |= {n: torch.full((i["x"].shape[2],), 7.0, device=DEV) for n in ("dd", "ddt_bias")}
    o["carry"], o["work"] = B.bload_scan_buffers(pos, i["x"], i["a"])
    return o


def call(pos, i, softplus=True, stream=None, o=None):
    o = fresh(pos, i) if o is None else o
    if i["z"] is None:
        o["dz"] = None
    more = {"d": i["d"], "dt_bias": i["dt_bias"], "z": i["z"], "softplus": softplus, "work": o["work"], "stream": stream}
    B.bload_scan(pos, i["x"], i["dt"], i["a"], i["b"], i["c"], o["y"], carry=o["carry"], **more)
    B.bload_scan_grad(pos, i["x"], i["dt"], i["a"], i["b"], i["c"], o["carry"], i["dy"], o["dx"], o["ddt"], o["da"], o["db"], o["dc"],
                      dd=o["dd"], ddt_bias=o["ddt_bias"], dz=o["dz"], **more)
    return o


def compare(o, blocks, i, softplus=True):
    torch.cuda.synchronize()
    val, tol = S.scan(blocks, i["x"], i["dt"], i["a"], i["b"], i["c"], i["d"], i["dt_bias"], i["z"], softplus, i["dy"])
    for n in FRAMES + SUMS:
        if n in val:
            L.close(o[n], val[n], tol[n], n)


CASES = [(F32, [[1]], 1, 1, 1), (BF, [[1], [-1]], 1, 8, 16), (FP, [[2, 3, 1], [6], [-6]], 6, 5, 3), (BF, [[15], [14, -1]], 15, 64, 16),
         (F32, [[16], [15, 1], [1, 15]], 16, 72, 8), (BF, [[17], [16, 1], [1, 16]], 17, 130, 16), (FP, [[300], [100, 150, 50], [1] * 300], 300, 40, 16),
         (F32, [[257], [-100, 157]], 257, 33, 5), (BF, [[200, -7]], 207, 24, 32), (F32, [[100, 33]], 133, 17, 31), (FP, [[90]], 90, 50, 64),
         (BF, [[64, 9]], 73, 16, 63), (F32, [[700, 1, 299]], 1000, 8, 16), (BF, [[1500]], 1500, 3, 7), (FP, [[1, 1, 1, 200]], 203, 200, 12)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%d-%d" % (str(c[0])[6:], c[2], c[3], c[4]))
@pytest.mark.parametrize("gated", [True, False])
def test_values_and_gradients(case, gated):
    dtype, blocks, t, c, n = case
    i = S.scan_inputs(len(blocks), t, c, n, dtype, 1, gated)
    compare(call(L.positions(t, blocks), i), blocks, i)


@pytest.mark.parametrize("seed", range(6))
def test_random_packings(seed):
    rng = np.random.default_rng(seed)
    t, c, nb = int(rng.integers(1, 900)), int(rng.integers(1, 150)), int(rng.integers(1, 5))
    blocks = L.random_blocks(rng, nb, t, [3.0, 40.0, 300.0][seed % 3])
    i = S.scan_inputs(nb, t, c, int(rng.integers(1, 65)), [BF, FP, F32][seed % 3], 50 * seed, bool(seed & 1))
    if seed & 2:
        i["d"] = None
    if seed & 4:
        i["dt_bias"] = None
    compare(call(L.positions(t, blocks), i), blocks, i)


def test_many_walks_in_one_piece_each_and_few_in_segments():
    """Both ways of cutting the work: 320 walks of four runs, and one of 160 runs."""
    blocks = [[30, 34], [64]] * 5
    i = S.scan_inputs(10, 64, 32 * 64, 16, BF, 3)
    compare(call(L.positions(64, blocks), i), blocks, i)
    for blocks in ([[2560]], [[128, 128, 1, 1000, 1303]], [[129, 2431]], [[-200, 1000, -360, 1000]]):
        i = S.scan_inputs(1, 2560, 20, 16, F32, 4)
        compare(call(L.positions(2560, blocks), i), blocks, i)


def test_without_softplus_and_with_growing_states():
    blocks, t = [[40, 24]], 64
    i = S.scan_inputs(1, t, 24, 8, F32, 9)
    i["dt"], i["dt_bias"] = i["dt"].abs() * 0.1, None
    i["a"][::2] *= -0.2  # exp(delta a) above 1
    compare(call(L.positions(t, blocks), i, softplus=False), blocks, i, softplus=False)


def test_steps_far_out():
    """softplus far on both sides: delta near 0 (nothing happens) and large (the state is forgotten)."""
    blocks, t = [[100, 28]], 128
    i = S.scan_inputs(1, t, 16, 8, F32, 10)
    i["dt"][0, ::3] = -60.0
    i["dt"][0, 1::3] = 40.0
    i["dt_bias"].zero_()
    compare(call(L.positions(t, blocks), i), blocks, i)


@pytest.mark.parametrize("junk", [math.nan, math.inf])
@pytest.mark.parametrize("t,c,blocks", [(400, 48, [[50, 70, -30, 200, -50]]), (3000, 16, [[500, 700, -300, 1400, -100]])])
def test_junk_on_padding_and_in_other_sequences_stays_there(junk, t, c, blocks):
    i = S.scan_inputs(1, t, c, 16, BF, 2)
    pos = L.positions(t, blocks)
    clean = call(pos, i)
    bad = pos < 0
    names = ("x", "dt", "b", "c", "z", "dy")
    for n in names:
        i[n][bad] = junk
    got = call(pos, i)
    torch.cuda.synchronize()
    for n in FRAMES + SUMS:
        assert torch.equal(got[n], clean[n]), n
    first, second = blocks[0][0], blocks[0][1]
    bad[0, first:first + second] = True
    for n in names:
        i[n][bad] = junk
    got = call(pos, i)
    torch.cuda.synchronize()
    for n in FRAMES + ("db", "dc"):
        assert torch.equal(got[n][~bad], clean[n][~bad]), n
        assert bool((got[n][pos < 0] == 0).all()), n


def test_strides_and_broadcast_inputs():
    blocks, t, c, n = [[90, 60]] * 3, 150, 64, 16
    pos = L.positions(t, blocks)
    i = S.scan_inputs(3, t, c, n, BF, 5)
    both = L.normal((3, t, 2 * c + 2 * n), BF, 5)  # a fused projection
    i["x"], i["z"], i["b"], i["c"] = both.split((c, c, n, n), -1)
    i["dy"] = L.normal((1, 1, c), BF, 6).expand(3, t, c)
    i["dt"] = i["dt"][:, :1].expand(3, t, c)
    o = fresh(pos, i)
    o["y"] = torch.full((t, 3, c), 7.0, dtype=BF, device=DEV).transpose(0, 1)
    grads = torch.full((3, t, 2 * c + 2 * n), 5.0, dtype=BF, device=DEV)
    o["dx"], o["dz"], o["db"], o["dc"] = grads.split((c, c, n, n), -1)
    compare(call(pos, i, o=o), blocks, i)
    i["x"] = L.normal((3, t, c + 3), BF, 7)[..., 3:]  # rows that start on any element
    i["b"] = L.normal((3, t, n + 1), BF, 8)[..., 1:]
    compare(call(pos, i), blocks, i)


def test_gradients_against_differences():
    blocks, t, c, n = [[40, 20, -4]], 64, 6, 5
    i = S.scan_inputs(1, t, c, n, F32, 3)
    o = call(L.positions(t, blocks), i)
    names = {"x": "dx", "dt": "ddt", "a": "da", "b": "db", "c": "dc", "d": "dd", "dt_bias": "ddt_bias", "z": "dz"}
    for name, grad in names.items():
        way = torch.randn(i[name].shape, dtype=torch.float64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
        ends = []
        for e in (1e-4, -1e-4):
            args = {k: i[k].double() + (e * way if k == name else 0) for k in names}
            ends.append(float((S.scan(blocks, **args)[0]["y"] * i["dy"].double()).sum()))
        slope = (ends[0] - ends[1]) / 2e-4
        assert abs(float((o[grad].double() * way).sum()) - slope) <= 1e-5 * float((o[grad].double() * way).abs().sum()), name


@pytest.mark.parametrize("t,c", [(1500, 200), (4000, 24)])
def test_repeated_calls_streams_and_graphs(t, c):
    rng = np.random.default_rng(2)
    blocks = L.random_blocks(rng, 2, t, 700.0)
    i = S.scan_inputs(2, t, c, 16, BF, 4)
    pos = L.positions(t, blocks)
    want, again = call(pos, i), call(pos, i)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    o, r = fresh(pos, i), fresh(pos, i)
    s.wait_stream(torch.cuda.current_stream())
    call(pos, i, stream=s, o=o)
    s.synchronize()
    with torch.cuda.graph(g):
        call(pos, i, o=r)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for n in FRAMES + SUMS + ("carry",):
        assert torch.equal(want[n], again[n]) and torch.equal(want[n], o[n]) and torch.equal(want[n], r[n]), n


def test_without_carry_and_sums_that_are_not_wanted():
    blocks, t = [[100, 29], [129]], 129
    i = S.scan_inputs(2, t, 40, 16, FP, 6)
    pos = L.positions(t, blocks)
    want = call(pos, i)
    y, o = torch.empty_like(i["x"]), fresh(pos, i)
    B.bload_scan(pos, i["x"], i["dt"], i["a"], i["b"], i["c"], y, i["d"], i["dt_bias"], i["z"], work=B.bload_scan_buffers(pos, i["x"], i["a"], gradient=False)[1])
    B.bload_scan_grad(pos, i["x"], i["dt"], i["a"], i["b"], i["c"], want["carry"], i["dy"], o["dx"], o["ddt"], o["da"], o["db"], o["dc"], i["d"],
                      None, i["dt_bias"], None, i["z"], o["dz"], work=o["work"])
    torch.cuda.synchronize()
    assert torch.equal(y, want["y"])
    for n in ("dx", "ddt", "dz", "da", "db", "dc"):
        assert torch.equal(o[n], want[n]), n


def test_rows_beyond_32_bits():
    c, far = 64, (1 << 31) + 64
    store = torch.empty(far + 64 * c, dtype=BF, device=DEV)
    x = torch.as_strided(store, (2, 50, c), (far, c, 1))
    x.copy_(L.normal((2, 50, c), BF, 3))
    blocks = [[50], [20, 30]]
    i = S.scan_inputs(2, 50, c, 16, BF, 7)
    i["x"] = x
    compare(call(L.positions(50, blocks), i), blocks, i)


@pytest.mark.parametrize("dtype,c,n", [(BF, 64, 16), (F32, 7, 5), (FP, 130, 64), (BF, 24, 20), (F32, 33, 1)])
@pytest.mark.parametrize("t,blocks", [(48, [[1, 5, -2, 40], [-3, 2, 43]]), (700, [[1, 500, 199], [-3, 350, 340]])])
def test_last_states_and_steps_go_on_where_a_packed_batch_ends(dtype, c, n, t, blocks):
    more, order = 3, [3, 0, 4, 1, 2]
    pos = L.positions(t, blocks)
    i = S.scan_inputs(2, t, c, n, dtype, 8)
    where = list(L.spans(blocks))
    ids, count = S.sequence_numbers(pos, torch.tensor(order, device=DEV))
    last = torch.full((count + 2, c, n), 5.0, device=DEV)  # two of other batches
    y = torch.empty_like(i["x"])
    _, work = B.bload_scan_buffers(pos, i["x"], i["a"], gradient=False)
    args = {"d": i["d"], "dt_bias": i["dt_bias"]}
    B.bload_scan(pos, i["x"], i["dt"], i["a"], i["b"], i["c"], y, z=i["z"], work=work, seq_id=ids, last=last, **args)
    torch.cuda.synchronize()
    val, tol = S.scan(blocks, i["x"], i["dt"], i["a"], i["b"], i["c"], z=i["z"], **args)
    L.close(y, val["y"], tol["y"], "y")
    assert bool((last[count:] == 5.0).all())
    L.close(last[torch.tensor(order, device=DEV)], val["last"], tol["last"], "last")
    state = last[:count].clone()
    e = S.scan_inputs(count, more, c, n, dtype, 9)  # three more frames of each
    want, bound = S.scan([[more]] * count, e["x"], e["dt"], i["a"], e["b"], e["c"], z=e["z"], start=state, **args)
    at = torch.zeros(count, dtype=torch.int32, device=DEV)
    for k, (_, s0, s1) in enumerate(where):
        at[order[k]] = s1 - s0
    for s in range(more):
        out = torch.empty((count, c), dtype=dtype, device=DEV)
        row = {k: e[k][:, s] for k in ("x", "dt", "b", "c", "z")}
        B.bload_scan_step(at + s, state, row["x"], row["dt"], i["a"], row["b"], row["c"], out, z=row["z"], **args)
        torch.cuda.synchronize()
        L.close(out, want["y"][:, s], bound["y"][:, s], "step %d" % s)
    L.close(state, want["last"], bound["last"], "state")


@pytest.mark.parametrize("n", [16, 6])
def test_steps_that_start_and_rows_without_a_frame(n):
    rows, c = 7, 36
    i = S.scan_inputs(rows, 1, c, n, BF, 3)
    e = {k: i[k][:, 0].clone() for k in ("x", "dt", "b", "c", "z")}
    state = L.normal((rows, c, n), F32, 4)
    clean = state.clone()
    state[0], state[3] = math.nan, math.inf  # what starts does not use them
    for k in e:
        e[k][1], e[k][4] = math.nan, math.inf  # nor does a row without a frame its inputs
    pos = torch.tensor([0, -1, 5, 0, -7, 1, 2], dtype=torch.int32, device=DEV)
    y, after, place, y2 = torch.empty((rows, c), dtype=BF, device=DEV), torch.full_like(state, 7.0), state.clone(), torch.empty((rows, c), dtype=BF, device=DEV)
    args = {"d": i["d"], "dt_bias": i["dt_bias"], "z": e["z"]}
    B.bload_scan_step(pos, state, e["x"], e["dt"], i["a"], e["b"], e["c"], y, next_state=after, **args)
    B.bload_scan_step(pos, place, e["x"], e["dt"], i["a"], e["b"], e["c"], y2, **args)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(after, place)
    start = torch.where((pos > 0)[:, None, None], clean, torch.zeros_like(clean))
    val, tol = S.scan([[1]] * rows, i["x"], i["dt"], i["a"], i["b"], i["c"], i["d"], i["dt_bias"], i["z"], start=start)
    frames = pos >= 0
    L.close(y[frames], val["y"][frames, 0], tol["y"][frames, 0], "y")
    L.close(after[frames], val["last"][frames], tol["last"][frames], "state")
    assert bool((y[~frames] == 0).all()) and torch.equal(after[~frames], state[~frames])


def test_no_blocks_and_refusals():
    x = torch.empty((0, 64, 16), device=DEV)
    pos = torch.empty((0, 64), dtype=torch.int32, device=DEV)
    i = S.scan_inputs(2, 200, 16, 4, F32, 1)
    carry, work = B.bload_scan_buffers(pos, x, i["a"])
    narrow = torch.empty((0, 64, 4), device=DEV)
    B.bload_scan(pos, x, x, i["a"], narrow, narrow, torch.empty_like(x), carry=carry, work=work)
    B.bload_scan_step(torch.empty(0, dtype=torch.int32, device=DEV), torch.empty((0, 16, 4), device=DEV), x[:, 0], x[:, 0], i["a"], narrow[:, 0],
                      narrow[:, 0], x[:, 0].clone())
    pos = L.positions(200, [[200], [100, 100]])
    o, ids = fresh(pos, i), S.sequence_numbers(pos)[0]
    X, DT, A, Bm, C, y = i["x"], i["dt"], i["a"], i["b"], i["c"], o["y"]
    last, at, state = torch.zeros((3, 16, 4), device=DEV), pos[:, 0].contiguous(), torch.zeros((2, 16, 4), device=DEV)
    run = {"work": o["work"]}
    for bad in (lambda: B.bload_scan(pos.short(), X, DT, A, Bm, C, y, **run), lambda: B.bload_scan(pos, X, DT.half(), A, Bm, C, y, **run),
                lambda: B.bload_scan(pos, X, DT, A.half(), Bm, C, y, **run), lambda: B.bload_scan(pos, X, DT, A, Bm[..., :3], C, y, **run),
                lambda: B.bload_scan(pos, X, DT, A[:, :3].contiguous(), Bm, C, y, **run), lambda: B.bload_scan(pos, X, DT, A, Bm, C, y, d=A, **run),
                lambda: B.bload_scan(pos, X, DT, A, Bm, C, y, last=last, **run), lambda: B.bload_scan(pos, X, DT, A, Bm, C, y, seq_id=ids, last=last.half(), **run),
                lambda: B.bload_scan(pos, X, DT, A, Bm, C, y, carry=o["carry"][:, :1], **run),
                lambda: B.bload_scan_grad(pos, X, DT, A, Bm, C, o["carry"], i["dy"], o["dx"], o["ddt"], o["da"], o["db"], o["dc"], z=i["z"], **run),
                lambda: B.bload_scan_step(at, state[:1], X[:, 0], DT[:, 0], A, Bm[:, 0], C[:, 0], y[:, 0]),
                lambda: B.bload_scan_step(at, state.half(), X[:, 0], DT[:, 0], A, Bm[:, 0], C[:, 0], y[:, 0])):
        with pytest.raises((TypeError, ValueError)):
            bad()
    wide = S.scan_inputs(2, 200, 16, 65, F32, 1)
    for bad, code in ((lambda: B.bload_scan(pos, X, DT, wide["a"], wide["b"], wide["c"], y, **run), -6),
                      (lambda: B.bload_scan(pos, X, DT, A, Bm, C, y[:, :1].expand(2, 200, 16), **run), -2),
                      (lambda: B.bload_scan_grad(pos, X, DT, A, Bm, C, None, i["dy"], o["dx"], o["ddt"], o["da"], o["db"], o["dc"], **run), -1),
                      (lambda: B.bload_scan_grad(pos, X, DT, A, Bm, C, o["carry"], i["dy"], o["dx"], o["ddt"], o["da"], o["db"], o["dc"]), -1),
                      (lambda: B.bload_scan_grad(pos, X, DT, A, Bm, C, o["carry"], i["dy"], o["dx"], o["ddt"], o["da"], o["db"], o["dc"],
                                                 work=o["work"][:256].clone()), -4)):
        with pytest.raises(B.BloadError) as e:
            bad()
        assert e.value.code == code


@pytest.mark.parametrize("dtype,c,n", [(BF, 2003, 16), (F32, 1999, 7), (FP, 1021, 24), (BF, 512, 64)])
def test_one_wave_of_walks_in_one_piece_each(dtype, c, n):
    """Between one and two walks for each of the machine's SMs, of many runs and an odd end; states of sequences that end in, at the end
    of and across runs, two calls alike."""
    blocks = [[203], [16, 32, 1, 100, 54], [-5, 150, 48], [31, 1, 171], [-203]]
    pos = L.positions(203, blocks)
    i = S.scan_inputs(5, 203, c, n, dtype, 12)
    ids, count = S.sequence_numbers(pos)
    args = {"d": i["d"], "dt_bias": i["dt_bias"], "z": i["z"]}
    _, work = B.bload_scan_buffers(pos, i["x"], i["a"], gradient=False)
    out = []
    for _ in range(2):
        y, last = torch.full_like(i["x"], 7.0), torch.full((count, c, n), 7.0, device=DEV)
        B.bload_scan(pos, i["x"], i["dt"], i["a"], i["b"], i["c"], y, work=work, seq_id=ids, last=last, **args)
        out.append((y, last))
    torch.cuda.synchronize()
    val, tol = S.scan(blocks, i["x"], i["dt"], i["a"], i["b"], i["c"], **args)
    L.close(out[0][0], val["y"], tol["y"], "y")
    L.close(out[0][1], val["last"], tol["last"], "last")
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
