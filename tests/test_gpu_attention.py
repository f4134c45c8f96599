"""bload_attention and its gradient against the definition in 64 bits, one sequence at a time."""
import math

import numpy as np
import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B

pytestmark = pytest.mark.gpu
DEV = L.DEV
BF, FP = torch.bfloat16, torch.float16


def buffers(q, k, v):
    b, t, h, _ = q.shape
    return dict(out=torch.full_like(q, 7.0), lse=torch.full((b, h, t), 7.0, device=DEV), dq=torch.full_like(q, 7.0),
                dk=torch.full_like(k, 7.0), dv=torch.full_like(v, 7.0), delta=torch.empty((b, h, t), device=DEV))


def call(pos, q, k, v, dout=None, stream=None, o=None, **how):
    o = buffers(q, k, v) if o is None else o
    B.bload_attention(pos, q, k, v, o["out"], o["lse"], stream=stream, **how)
    if dout is not None:
        B.bload_attention_grad(pos, q, k, v, o["out"], o["lse"], dout, o["dq"], o["dk"], o["dv"], o["delta"], stream=stream, **how)
    return o


def compare(o, blocks, q, k, v, dout=None, **how):
    torch.cuda.synchronize()
    val, tol = L.attention(blocks, q, k, v, dout, **how)
    empty = torch.isinf(val["lse"])
    assert bool((o["lse"][empty] == -math.inf).all())
    L.close(o["lse"][~empty], val["lse"][~empty], tol["lse"][~empty], "lse")
    for n in ("out",) if dout is None else ("out", "dq", "dk", "dv"):
        L.close(o[n], val[n], tol[n], n)
    return val, tol


def inputs(b, t, h, hk, d, dtype, seed=1):
    return (L.normal((b, t, h, d), dtype, seed, std=1.5), L.normal((b, t, hk, d), dtype, seed + 1),
            L.normal((b, t, hk, d), dtype, seed + 2), L.normal((b, t, h, d), dtype, seed + 3))


def slopes_of(h):
    return torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device=DEV)


# dtype, blocks (lengths; negative = padding), t, heads, key heads, head size, causal, window, cap, slopes
CASES = [
    (BF, [[1]], 1, 1, 1, 64, True, 0, 0.0, False),
    (FP, [[1], [-1]], 1, 3, 1, 8, False, 0, 0.0, False),
    (BF, [[2, 3, 4, 5], [6, 6], [-14]], 14, 2, 2, 64, True, 0, 0.0, False),
    (FP, [[64], [30, 30, -4], [1] * 64], 64, 8, 4, 64, True, 0, 0.0, False),
    (BF, [[64], [30, 30, -4], [1] * 64], 64, 4, 4, 128, False, 0, 0.0, False),
    (BF, [[127], [126, -1]], 127, 2, 1, 128, True, 0, 0.0, False),
    (FP, [[128], [127, 1], [1, 127], [64, 64]], 128, 2, 1, 128, True, 0, 0.0, False),
    (BF, [[129], [128, 1], [1, 128], [129]], 129, 2, 2, 64, False, 0, 0.0, False),
    (BF, [[191, 1, 65], [256, -1], [100, 100, 57]], 257, 4, 2, 128, True, 0, 0.0, False),
    (FP, [[191, 1, 65], [256, -1], [100, 100, 57]], 257, 4, 1, 64, False, 0, 0.0, False),
    (BF, [[1000], [200, 300, 450, -50], [5, 900, 95]], 1000, 2, 1, 64, True, 0, 0.0, False),
    (BF, [[1000], [200, 300, 450, -50], [5, 900, 95]], 1000, 2, 1, 128, False, 0, 0.0, False),
    (BF, [[700, 201], [901]], 901, 2, 2, 80, True, 0, 30.0, False),
    (FP, [[700, 201], [901]], 901, 2, 2, 96, False, 0, 50.0, True),
    (BF, [[700, 201], [901]], 901, 4, 2, 120, True, 0, 0.0, True),
    (BF, [[513, 130]], 643, 2, 1, 128, True, 1, 0.0, False),
    (BF, [[513, 130]], 643, 2, 1, 128, True, 100, 0.0, False),
    (FP, [[513, 130]], 643, 2, 1, 64, False, 65, 0.0, True),
    (BF, [[513, 130]], 643, 2, 1, 64, False, 129, 20.0, True),
    (BF, [[513, 130]], 643, 2, 1, 16, True, 10000, 0.0, False),
    (FP, [[-300, 40, -160, 100]], 600, 2, 1, 24, True, 0, 0.0, False),
    (BF, [[-300, 40, -160, 100]], 600, 2, 1, 72, False, 0, 0.0, False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%dx%dx%d%s%s%s%s" % (
    str(c[0])[6:], c[2], c[3], c[4], c[5], "-causal" if c[6] else "", "-w%d" % c[7] if c[7] else "", "-cap" if c[8] else "",
    "-bias" if c[9] else ""))
def test_values_and_gradients(case):
    dtype, blocks, t, h, hk, d, causal, window, cap, bias = case
    q, k, v, dout = inputs(len(blocks), t, h, hk, d, dtype)
    how = dict(causal=causal, window=window, softcap=cap, slopes=slopes_of(h) if bias else None)
    compare(call(L.positions(t, blocks), q, k, v, dout, **how), blocks, q, k, v, dout, **how)


@pytest.mark.parametrize("seed", range(8))
def test_random_packings(seed):
    rng = np.random.default_rng(seed)
    t, d = int(rng.integers(1, 900)), 8 * int(rng.integers(1, 17))
    hk, g, nb = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(1, 4))
    blocks = L.random_blocks(rng, nb, t, [3.0, 30.0, 200.0, 2000.0][seed % 4])
    dtype = [BF, FP][seed % 2]
    q, k, v, dout = inputs(nb, t, hk * g, hk, d, dtype, 100 * seed)
    how = dict(causal=bool(rng.random() < 0.6), window=int(rng.choice([0, 0, 7, 150])), softcap=float(rng.choice([0.0, 0.0, 25.0])),
               slopes=slopes_of(hk * g) if rng.random() < 0.4 else None, scale=float(rng.choice([0.07, 0.2])))
    compare(call(L.positions(t, blocks), q, k, v, dout, **how), blocks, q, k, v, dout, **how)


def test_long_sequence():
    blocks = [[20011, 3, 2000]]
    q, k, v, dout = inputs(1, 22100, 1, 1, 64, BF)
    how = dict(causal=True)
    compare(call(L.positions(22100, blocks), q, k, v, dout, **how), blocks, q, k, v, dout, **how)


def test_longest_block_with_a_window():
    blocks = [[100, 32668]]
    q, k, v, dout = inputs(1, 32768, 1, 1, 64, FP)
    how = dict(causal=True, window=300)
    o = call(L.positions(32768, blocks), q, k, v, dout, **how)
    # the definition over the last 2,000 queries, which see nothing before slot 30,000
    part = slice(30000, 32768)
    val, tol = L.attention([[2768]], q[:, part], k[:, part], v[:, part], dout[:, part], **how)
    last = slice(768, 2768)
    L.close(o["out"][:, part][:, last], val["out"][:, last], tol["out"][:, last], "out")
    L.close(o["dq"][:, part][:, last], val["dq"][:, last], tol["dq"][:, last], "dq")
    L.close(o["dk"][:, part][:, last], val["dk"][:, last], tol["dk"][:, last], "dk")


@pytest.mark.parametrize("layout", ["fused", "heads_first", "rows_apart"])
def test_layouts(layout):
    blocks, t, h, hk, d = [[150, 50], [199, -1]], 200, 4, 2, 64
    nb = len(blocks)
    if layout == "fused":
        qkv = L.normal((nb, t, h + 2 * hk, d), BF, 3)
        q, k, v = qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:]
        grads = torch.full_like(qkv, 3.0)
        outs = dict(dq=grads[:, :, :h], dk=grads[:, :, h:h + hk], dv=grads[:, :, h + hk:])
        dout = L.normal((nb, t, h, d), BF, 4)
    elif layout == "heads_first":
        mk = lambda n, s: L.normal((nb, n, t, d), BF, s).transpose(1, 2)  # noqa: E731
        q, k, v, dout = mk(h, 1), mk(hk, 2), mk(hk, 3), mk(h, 4)
        outs = {}
    else:
        mk = lambda n, s: L.normal((nb + 1, t + 3, n + 1, d + 8), BF, s)[1:, 3:, 1:, 8:]  # noqa: E731
        q, k, v, dout = mk(h, 1), mk(hk, 2), mk(hk, 3), mk(h, 4)
        outs = dict(dq=mk(h, 5), dk=mk(hk, 6), dv=mk(hk, 7), out=mk(h, 8))
    o = buffers(q, k, v)
    o.update(outs)
    around = {n: x._base.clone() for n, x in outs.items()} if layout == "rows_apart" else {}
    compare(call(L.positions(t, blocks), q, k, v, dout, o=o), blocks, q, k, v, dout)
    for n, was in around.items():  # nothing outside the tensors was written
        now = outs[n]._base.clone()
        now[1:, 3:, 1:, 8:] = was[1:, 3:, 1:, 8:]
        assert torch.equal(now, was), n


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("junk", [math.nan, math.inf, -math.inf, 6.0e4])
@pytest.mark.parametrize("causal", [True, False])
def test_what_hidden_slots_hold_has_no_influence(junk, causal, d):
    """Padding full of junk, and a sequence full of junk beside clean ones: the clean sequences' results are those of a
    batch without it, and padding gives zeros."""
    blocks, t = [[50, 70, 200, 30, -50], [40, -60, 300]], 400
    pos = L.positions(t, blocks)
    q, k, v, dout = inputs(2, t, 4, 2, d, FP)
    clean = call(pos, q, k, v, dout, causal=causal)
    clean = {n: x.clone() for n, x in clean.items()}
    bad = torch.zeros((2, t), dtype=torch.bool, device=DEV)
    bad[0, 350:] = True
    bad[0, 50:120] = True  # the sequence of 70
    bad[1, 40:100] = True
    for x in (q, k, v, dout):
        x[bad] = junk
    got = call(pos, q, k, v, dout, causal=causal)
    torch.cuda.synchronize()
    for n in ("out", "dq", "dk", "dv"):
        L.close(got[n][~bad], clean[n][~bad].double(), 0.02 + 0.02 * clean[n][~bad].double().abs(), n)
        assert bool((got[n][pos < 0] == 0).all()), n
    assert bool((got["lse"].transpose(1, 2)[pos < 0] == -math.inf).all())


def test_junk_in_the_future_stays_there():
    """Causal: keys and values of one slot are infinite or NaN; slots before it do not notice, slots after it do."""
    blocks, t, at = [[300]], 300, 170
    q, k, v, dout = inputs(1, t, 2, 2, 64, BF)
    pos = L.positions(t, blocks)
    v2, k2 = v.clone(), k.clone()
    v2[0, at] = math.nan
    k2[0, at] = math.inf
    clean, got = call(pos, q, k, v), call(pos, q, k2, v2)
    torch.cuda.synchronize()
    L.close(got["out"][:, :at], clean["out"][:, :at].double(), 0.01 + 0.01 * clean["out"][:, :at].double().abs(), "out")
    assert bool(torch.isnan(got["out"][0, at:]).all())


def test_extreme_scores():
    """Scores far apart and all far from zero: the running maximum keeps every exponential in range."""
    blocks, t = [[400]], 400
    q, k, v, dout = inputs(1, t, 2, 1, 64, BF)
    for shift in (0.0, 40.0, -40.0):
        qq = (q.float() * 8 + shift).to(BF)
        kk = (k.float() * 4 + 1.0).to(BF)
        compare(call(L.positions(t, blocks), qq, kk, v, dout), blocks, qq, kk, v, dout)
    up = torch.linspace(0, 60, t, device=DEV)[None, :, None, None]  # scores that rise along the keys: the maximum moves in every tile
    kk = (k.float() * 0.1 + up / 8).to(BF)
    qq = torch.ones_like(q)
    compare(call(L.positions(t, blocks), qq, kk, v, dout, causal=False), blocks, qq, kk, v, dout, causal=False)


def test_gradients_against_differences():
    blocks, t, h, hk, d = [[40, 24], [50, -14]], 64, 4, 2, 32
    q, k, v, dout = inputs(2, t, h, hk, d, FP)
    how = dict(softcap=8.0, slopes=slopes_of(h), window=30)
    o = call(L.positions(t, blocks), q, k, v, dout, **how)
    _, tol = L.attention(blocks, q, k, v, dout, **how)

    base = [x.double() for x in (q, k, v)]
    for n, (name, x) in enumerate(zip(("dq", "dk", "dv"), base)):
        way = torch.randn(x.shape, dtype=torch.float64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(n))
        ends = []
        for e in (1e-4, -1e-4):
            args = list(base)
            args[n] = x + e * way
            ends.append(float((L.attention(blocks, *args, **how)[0]["out"] * dout.double()).sum()))
        slope = (ends[0] - ends[1]) / 2e-4
        assert abs(float((o[name].double() * way).sum()) - slope) <= float((tol[name] * way.abs()).sum()) + 1e-5 * abs(slope), name


def test_repeated_calls_are_identical():
    rng = np.random.default_rng(0)
    blocks = L.random_blocks(rng, 2, 1500, 120.0)
    q, k, v, dout = inputs(2, 1500, 4, 2, 64, BF)
    pos = L.positions(1500, blocks)
    one, two = call(pos, q, k, v, dout), call(pos, q, k, v, dout)
    for n in one:
        assert torch.equal(one[n], two[n]), n


def test_without_lse_and_on_another_stream_and_from_a_graph():
    blocks, t = [[100, 29], [129]], 129
    q, k, v, dout = inputs(2, t, 2, 2, 64, BF)
    pos = L.positions(t, blocks)
    want = call(pos, q, k, v, dout)
    out = torch.empty_like(q)
    B.bload_attention(pos, q, k, v, out)
    torch.cuda.synchronize()
    assert torch.equal(out, want["out"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = buffers(q, k, v)
    s.wait_stream(torch.cuda.current_stream())
    call(pos, q, k, v, dout, stream=s, o=got)
    s.synchronize()
    for n in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(got[n], want[n]), n
    g, o = torch.cuda.CUDAGraph(), buffers(q, k, v)
    with torch.cuda.graph(g):
        call(pos, q, k, v, dout, o=o)
    for x in o.values():
        x.fill_(3.0)
    g.replay()
    torch.cuda.synchronize()
    for n in ("out", "lse", "dq", "dk", "dv"):
        assert torch.equal(o[n], want[n]), n


def test_no_blocks():
    q = torch.empty((0, 64, 2, 64), dtype=BF, device=DEV)
    pos = torch.empty((0, 64), dtype=torch.int32, device=DEV)
    lse = torch.empty((0, 2, 64), device=DEV)
    B.bload_attention(pos, q, q, q, torch.empty_like(q), lse)
    B.bload_attention_grad(pos, q, q, q, q, lse, q, torch.empty_like(q), torch.empty_like(q), torch.empty_like(q), lse)
    torch.cuda.synchronize()


def test_positions_of_a_plan():
    """The positions as bload_pack writes them, against those laid out by hand from the plan's tables."""
    lengths = torch.tensor([5, 64, 17, 33, 40, 9, 60, 2], dtype=torch.int32, device=DEV)
    plan = B.bload_plan(lengths, 64, 7)
    pos = torch.empty((plan.n_blocks, 64), dtype=torch.int32, device=DEV)
    B.bload_pack(plan, None, 1, 0, plan.n_blocks, pos=pos)
    tab = {k: x.cpu().numpy() for k, x in plan.tables().items()}
    blocks = [[int(lengths[tab["seg_seq"][s]]) for s in range(tab["block_seg_begin"][b], tab["block_seg_begin"][b + 1])]
              for b in range(plan.n_blocks)]
    assert torch.equal(pos, L.positions(64, blocks))
    q, k, v, dout = inputs(plan.n_blocks, 64, 2, 1, 64, BF)
    compare(call(pos, q, k, v, dout), blocks, q, k, v, dout)


def test_refusals():
    blocks, t = [[60, 4]], 64
    q, k, v, dout = inputs(1, t, 4, 2, 64, BF)
    pos = L.positions(t, blocks)
    out, lse = torch.empty_like(q), torch.empty((1, 4, t), device=DEV)

    def refused(kind, *args, **how):
        with pytest.raises(kind) as e:
            B.bload_attention(*args, **how)
        return getattr(e.value, "code", None)

    assert refused(TypeError, pos.long(), q, k, v, out) is None
    assert refused(TypeError, pos.cpu(), q, k, v, out) is None
    assert refused(ValueError, pos, q, k, v, out[:, :63]) is None
    assert refused(TypeError, pos, q, k.half(), v, out) is None
    assert refused(TypeError, pos, q, k, v, out, lse.half()) is None
    assert refused(ValueError, pos, q.transpose(2, 3), k, v, out) is None
    f = lambda x: x.float()  # noqa: E731
    assert refused(B.BloadError, pos, f(q), f(k), f(v), f(out)) == -6
    assert refused(B.BloadError, pos, q[..., :60], k[..., :60], v[..., :60], out[..., :60]) == -6
    assert refused(B.BloadError, pos, q[:, :, :3], k, v, out[:, :, :3]) == -2  # 3 heads on 2
    assert refused(B.BloadError, pos, q, k, v, out, window=-1) == -2
    assert refused(B.BloadError, pos, q, k, v, out, softcap=-1.0) == -2
    assert refused(B.BloadError, pos, q, k, v, out, scale=math.nan) == -2
    assert refused(B.BloadError, pos, q[:, :, :1].expand(1, t, 4, 64), k, v, out) == -2  # broadcast heads: use kv_heads
    odd = torch.empty(q.numel() + 8, dtype=BF, device=DEV)[4:4 + q.numel()].view_as(q)
    assert refused(B.BloadError, pos, odd, k, v, out) == -5
    with pytest.raises(B.BloadError) as e:
        wide = torch.empty((1, t, 4, 68), dtype=BF, device=DEV)[..., :64]
        B.bload_attention(pos, wide, k, v, out)
    assert e.value.code == -5
