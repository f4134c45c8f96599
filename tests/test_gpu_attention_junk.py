"""Attention over batches in which frames hold infinities and NaN: what may see them shows them, all else is as if they
were not there."""
import math

import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B
from test_gpu_attention import BF, FP, buffers, call, inputs, slopes_of

pytestmark = pytest.mark.gpu
DEV = L.DEV


def without(blocks, bad):
    """The packing with the sequences of `bad` ({(block, index)}) as padding."""
    return [[-n if n > 0 and (b, k) in bad else n for k, n in enumerate(here)] for b, here in enumerate(blocks)]


def slots(blocks, t, bad):
    """bool [blocks, t]: slots of the sequences of `bad`."""
    m = torch.zeros((len(blocks), t), dtype=torch.bool, device=DEV)
    for b, here in enumerate(blocks):
        s = 0
        for k, n in enumerate(here):
            m[b, s:s + abs(n)] |= (b, k) in bad
            s += abs(n)
    return m


def compare_clean(got, blocks, t, bad, q, k, v, dout, **how):
    """Everything outside the sequences of `bad`, against the definition of the batch without them."""
    torch.cuda.synchronize()
    here = ~slots(blocks, t, bad)
    zero = {n: x.masked_fill(~here[..., None, None], 0.0) for n, x in (("q", q), ("k", k), ("v", v), ("dout", dout))}
    val, tol = L.attention(without(blocks, bad), zero["q"], zero["k"], zero["v"], zero["dout"], **how)
    frame = ~torch.isinf(val["lse"])
    L.close(got["lse"][frame], val["lse"][frame], tol["lse"][frame], "lse")
    for n in ("out", "dq", "dk", "dv"):
        L.close(got[n][here], val[n][here], tol[n][here], n)


@pytest.mark.parametrize("d", [24, 64, 128])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_walks_of_a_single_tile_end_in_order(dtype, d):
    """Every CTA meets junk in the only tile of its walk, call after call: its products and copies have to have ended
    before the next CTA takes its place."""
    t, nb, h, hk = 40, 300, 4, 2
    blocks = [[3, 1, 7, 2, 9, 4, 12, -2]] * nb
    bad = {(b, k) for b in range(nb) for k in (1, 4)}
    q, k, v, dout = inputs(nb, t, h, hk, d, dtype)
    for x in (q, k, v, dout):
        x[slots(blocks, t, bad)] = math.nan
    pos = L.positions(t, blocks)
    first = {n: x.clone() for n, x in call(pos, q, k, v, dout).items()}
    for _ in range(20):
        again = call(pos, q, k, v, dout)
        for n in first:
            assert torch.equal(first[n].nan_to_num(7.0), again[n].nan_to_num(7.0)), n
    assert B.bload_device_timeouts() == 0
    few = {n: x[:8] for n, x in first.items()}
    compare_clean(few, blocks[:8], t, {x for x in bad if x[0] < 8}, q[:8], k[:8], v[:8], dout[:8])


# dtype, head size, causal, window, cap, slopes
HOWS = [(BF, 64, True, 0, 0.0, False), (FP, 128, True, 0, 0.0, False), (BF, 88, True, 0, 30.0, True), (FP, 88, False, 0, 20.0, True),
        (FP, 24, False, 70, 0.0, True), (BF, 128, True, 90, 8.0, False), (FP, 64, False, 0, 0.0, False), (BF, 120, False, 150, 0.0, False)]
NAMES = ["%s-%d%s%s%s%s" % (str(c[0])[6:], c[1], "-causal" if c[2] else "", "-w%d" % c[3] if c[3] else "", "-cap" if c[4] else "",
                            "-bias" if c[5] else "") for c in HOWS]


@pytest.mark.parametrize("case", HOWS, ids=NAMES)
def test_clean_sequences_keep_their_bits(case):
    """Sequences full of junk, and junk on padding, beside clean sequences in the same 128 rows and in the tiles of their walks."""
    dtype, d, causal, window, cap, bias = case
    blocks, t, h, hk = [[50, 70, 200, 30, -50], [40, -60, 300], [300, 20, 80], [9] * 44 + [-4]], 400, 4, 2
    bad = {(0, 1), (0, 4), (1, 1), (2, 0), (3, 3), (3, 30)}
    how = dict(causal=causal, window=window, softcap=cap, slopes=slopes_of(h) if bias else None)
    pos = L.positions(t, blocks)
    q, k, v, dout = inputs(len(blocks), t, h, hk, d, dtype)
    clean = {n: x.clone() for n, x in call(pos, q, k, v, dout, **how).items()}
    here = slots(blocks, t, bad)
    for which, junk in (("qkvo", math.nan), ("v", math.inf), ("o", -math.inf), ("kq", math.inf), ("qkvo", 3.0e4)):
        x = dict(q=q.clone(), k=k.clone(), v=v.clone(), o=dout.clone())
        for n in which:
            x[n][here] = junk
        got = call(pos, x["q"], x["k"], x["v"], x["o"], **how)
        torch.cuda.synchronize()
        for n in ("out", "dq", "dk", "dv"):
            assert torch.equal(got[n][~here], clean[n][~here]), (which, junk, n)
            assert bool((got[n][pos < 0] == 0).all()), (which, junk, n)
        assert torch.equal(got["lse"].transpose(1, 2)[~here], clean["lse"].transpose(1, 2)[~here]), (which, junk)
        compare_clean(got, blocks, t, bad, x["q"], x["k"], x["v"], x["o"], **how)


def seen(t, s0, s1, causal, window):
    """bool [t, t]: query i of the sequence [s0, s1) may see key j."""
    i = torch.arange(t, device=DEV)
    apart = i[:, None] - i[None, :]
    ok = ((i >= s0) & (i < s1))[:, None] & ((i >= s0) & (i < s1))[None, :]
    if causal:
        ok &= apart >= 0
    if window:
        ok &= apart.abs() < window
    return ok


@pytest.mark.parametrize("case", HOWS, ids=NAMES)
def test_who_sees_a_bad_element_shows_it(case):
    """Single infinities and NaN in v (dout): by the formula they reach that element of out (dv) of every row that sees the frame, with
    their sign, and of no other.  A bad element of dout also reaches all of its own dq, and of dk where it is seen."""
    dtype, d, causal, window, cap, bias = case
    t, h, hk, s0 = 420, 2, 1, 20  # the sequence lies across three tiles
    blocks = [[s0, t - s0 - 30, 30]]
    how = dict(causal=causal, window=window, softcap=cap, slopes=0.1 * slopes_of(h) if bias else None, scale=0.05)
    pos = L.positions(t, blocks)
    q, k, v, dout = inputs(1, t, h, hk, d, dtype)
    at = [(25, 0, math.inf), (100, d - 1, -math.inf), (127, 8, math.nan), (128, 3, math.inf), (200, 3, -math.inf), (300, 5, math.inf), (389, 1, math.nan)]
    ok = seen(t, s0, t - 30, causal, window)
    clean = {n: x.clone() for n, x in call(pos, q, k, v, dout, **how).items()}

    def expected(n, head, rows_see, x, xh):  # `x` has the junk, in head xh; rows_see [rows, slots]
        want = clean[n][0, :, head].clone()
        for s, e, _ in at:
            want[rows_see[:, s], e] = want[rows_see[:, s], e] + x[0, s, xh, e]  # finite + infinite, or NaN
        return want

    bad = v.clone()
    for s, e, j in at:
        bad[0, s, 0, e] = j
    got = call(pos, q, k, bad, **how)
    torch.cuda.synchronize()
    assert torch.equal(got["lse"], clean["lse"])
    for head in range(h):
        want, mine = expected("out", head, ok, bad, 0), got["out"][0, :, head]
        touched = torch.zeros_like(want, dtype=torch.bool)
        for s, e, _ in at:
            touched[ok[:, s], e] = True
        assert torch.equal(mine[~touched], clean["out"][0, :, head][~touched])  # what is not touched keeps its bits
        assert torch.equal(mine[touched].nan_to_num(7.0, 8.0, 9.0), want[touched].nan_to_num(7.0, 8.0, 9.0))

    bad = dout.clone()
    for s, e, j in at:
        bad[0, s, 1, e] = j  # of one of the two heads that share the keys
    got = call(pos, q, k, v, bad, **how)
    torch.cuda.synchronize()
    sees = torch.zeros(t, dtype=torch.bool, device=DEV)  # keys that a bad query sees
    own = torch.zeros(t, dtype=torch.bool, device=DEV)
    for s, _, _ in at:
        sees |= ok[s]
        own[s] = True
    want, mine = expected("dv", 0, ok.T, bad, 1), got["dv"][0, :, 0]
    touched = torch.zeros_like(want, dtype=torch.bool)
    for s, e, _ in at:
        touched[ok[s], e] = True
    assert torch.equal(mine[~touched], clean["dv"][0, :, 0][~touched])
    assert torch.equal(mine[touched].nan_to_num(7.0, 8.0, 9.0), want[touched].nan_to_num(7.0, 8.0, 9.0))
    assert torch.equal(got["dk"][0, ~sees], clean["dk"][0, ~sees]) and not bool(torch.isfinite(got["dk"][0, sees]).any())
    assert torch.equal(got["dq"][0, ~own], clean["dq"][0, ~own]) and not bool(torch.isfinite(got["dq"][0, own, 1]).any())
    assert torch.equal(got["dq"][0, own, 0], clean["dq"][0, own, 0])


@pytest.mark.parametrize("d", [64, 128])
def test_a_bad_key_reaches_every_row_that_sees_it(d):
    t, blocks = 300, [[40, 200, 60]]
    pos, at = L.positions(t, blocks), 150
    q, k, v, dout = inputs(1, t, 2, 1, d, BF)
    clean = {n: x.clone() for n, x in call(pos, q, k, v, dout).items()}
    k[0, at, 0, 3] = math.nan
    got = call(pos, q, k, v, dout)
    torch.cuda.synchronize()
    hit = slice(at, 240)  # the rest of its sequence
    for n in ("out", "dq"):
        assert bool(torch.isnan(got[n][0, hit]).all()), n
        for part in (slice(0, at), slice(240, t)):
            assert torch.equal(got[n][0, part], clean[n][0, part]), n
    for n in ("dk", "dv"):  # through those rows' weights, every key of the sequence
        assert bool(torch.isnan(got[n][0, 40:240]).all()), n
        for part in (slice(0, 40), slice(240, t)):
            assert torch.equal(got[n][0, part], clean[n][0, part]), n


@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_gradients_that_overflowed_everywhere(dtype):
    """What a loss scale that is too large leaves: infinities and NaN all over dout.  Nothing finite comes back for a frame, zeros
    for padding, and the call comes to an end."""
    t, blocks = 2000, [[700, 1, 900, -99, 300], [2000]]
    pos = L.positions(t, blocks)
    q, k, v, dout = inputs(2, t, 4, 2, 64, dtype)
    dout = torch.where(dout > 0, math.inf, math.nan).to(dtype)
    got = call(pos, q, k, v, dout)
    torch.cuda.synchronize()
    for n in ("dq", "dk", "dv"):
        assert not bool(torch.isfinite(got[n][pos >= 0]).any()), n
        assert bool((got[n][pos < 0] == 0).all()), n
    assert B.bload_device_timeouts() == 0
