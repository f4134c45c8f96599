"""Attention's dq for rows that see few keys: the error of the rounded out in dout . out must not show, whatever else is packed
into the same block.

The keys' values share a large part, so dout . v_j - delta is small against dout . out, and a delta taken from the rounded
out is off by a fifth of it.  Bound: with delta' = delta - x from the rounded out, |x| <= e_x, the kernel forms dS' = P (dP - delta'), rounds
it to 16 bits, and takes x sum_j P_ij inner k_j off again, with P inner rounded to 16 bits; so beside u |dS| no more is left of x than 2 u P e_x."""
import math

import pytest
import torch

import layer_util as L
from test_gpu_attention import BF, FP, call, slopes_of

pytestmark = pytest.mark.gpu
DEV, E = L.DEV, L.E
SHORT = 1024  # keys that a row may see for the bound to hold


def expected(blocks, q, k, v, dout, scale, softcap, slopes, causal, window):
    """(dq, allowed error, delta, allowed error, rows that see at most SHORT keys), float64."""
    u, tiny = L.U[q.dtype], (2.0 ** -24 if q.dtype == FP else 2.0 ** -126)
    nb, t, h, d = q.shape
    dq, t_dq = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    dl, t_dl = (torch.zeros((nb, h, t), dtype=torch.float64, device=DEV) for _ in range(2))
    few = torch.ones((nb, t), dtype=torch.bool, device=DEV)
    for b, s0, s1 in L.spans(blocks):
        i = torch.arange(s1 - s0, device=DEV)
        apart = (i[:, None] - i[None, :]).abs()
        ok = torch.ones_like(apart, dtype=torch.bool)
        if causal:
            ok &= i[:, None] >= i[None, :]
        if window:
            ok &= apart < window
        few[b, s0:s1] = ok.sum(-1) <= SHORT
        for head in range(h):
            kv = head // (h // k.shape[2])
            Q, K, V, G = (x.double() for x in (q[b, s0:s1, head], k[b, s0:s1, kv], v[b, s0:s1, kv], dout[b, s0:s1, head]))
            raw, size = scale * (Q @ K.T), abs(scale) * (Q.abs() @ K.abs().T)
            s, inner = raw, torch.ones_like(raw)
            if softcap:
                th = torch.tanh(raw / softcap)
                s, inner = softcap * th, 1 - th * th
            bias = 0.0 if slopes is None else float(slopes[head]) * apart.double()
            P = torch.softmax((s - bias).masked_fill(~ok, -math.inf), -1)
            mag = torch.where(ok, size + (abs(bias) if slopes is not None else 0.0) + softcap, 0.0).amax(-1, keepdim=True)
            e_p = 2 * ((d + 8) * E * torch.where(ok, size, 0.0).amax(-1, keepdim=True) + 16 * E * mag + 16 * E)  # relative, of P
            out, dP = P @ V, G @ V.T
            delta = (P * dP).sum(-1, keepdim=True)
            e_x = (G.abs() * (u * out.abs() + (1.05 * u + e_p) * (P @ V.abs()) + tiny * (1 + V.abs().sum(0)))).sum(-1, keepdim=True)
            e_dp = (d + 8) * E * (G.abs() @ V.abs().T)
            # of P (dP - delta'), in 32 bits: its own error, and that of its sum over j (rounding of a sum of n terms: n E)
            e_g = P * (2 * e_p * ((dP - delta).abs() + e_x) + e_dp)
            e_sum = e_g.sum(-1, keepdim=True) + len(i) * E * (P * ((dP - delta).abs() + e_x)).sum(-1, keepdim=True)
            dS = P * (dP - delta) * inner
            e_ds = 1.05 * u * (dS.abs() + 2 * P * e_x * inner) + e_g * inner + P * inner * e_sum + P * ((dP - delta).abs() + e_x) * (64 * E + 2 * e_p * (softcap > 0)) + \
                tiny * ok * (1 + (dP - delta).abs() + e_x)
            dq[b, s0:s1, head] = scale * (dS @ K)
            t_dq[b, s0:s1, head] = abs(scale) * (e_ds @ K.abs())
            dl[b, head, s0:s1], t_dl[b, head, s0:s1] = delta[:, 0], (e_sum + 4 * E * (delta.abs() + e_x))[:, 0]
    t_dq += u * dq.abs() + tiny
    return dq, t_dq + 64 * E * t_dq / u, dl, t_dl, few


MIXED = [[1500, 20, 60, 5, 443], [3, 1400, 7, 100, 538], [1800, 1, 1, 1, 30, -20, 195]]
CASES = [  # dtype, head size, blocks, t, causal, window, cap, slopes
    (BF, 16, MIXED, 2048, True, 0, 0.0, False), (FP, 72, MIXED, 2048, True, 0, 0.0, False), (BF, 72, MIXED, 2048, False, 0, 0.0, True),
    (FP, 24, MIXED, 2048, False, 0, 0.0, False), (BF, 128, MIXED, 2048, True, 0, 20.0, True), (BF, 64, [[40, 60, 27], [127]], 127, True, 0, 0.0, False),
    (BF, 24, [[1024], [1000, 24]], 1024, True, 0, 0.0, False), (BF, 72, [[50, 1950]], 2000, True, 60, 0.0, False), (FP, 40, [[1500, 500]], 2000, False, 512, 0.0, False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%d-%d%s%s%s%s" % (str(c[0])[6:], c[1], c[3], "-causal" if c[4] else "",
                                                                             "-w%d" % c[5] if c[5] else "", "-cap" if c[6] else "", "-bias" if c[7] else ""))
def test_rows_with_few_keys(case):
    dtype, d, blocks, t, causal, window, cap, bias = case
    nb, h, hk = len(blocks), 2, 1
    q, dout = L.normal((nb, t, h, d), dtype, 1), L.normal((nb, t, h, d), dtype, 4)
    k, v = L.normal((nb, t, hk, d), dtype, 2, mean=1.0), L.normal((nb, t, hk, d), dtype, 3, mean=8.0, std=0.25)
    how = dict(causal=causal, window=window, softcap=cap, slopes=0.1 * slopes_of(h) if bias else None, scale=d ** -0.5)
    got = call(L.positions(t, blocks), q, k, v, dout, **how)
    torch.cuda.synchronize()
    dq, t_dq, delta, t_delta, few = expected(blocks, q, k, v, dout, **how)
    assert int(few.sum()) > 100
    L.close(got["dq"][few], dq[few], t_dq[few], "dq")
    L.close(got["delta"], delta, t_delta, "delta")


def test_a_row_does_not_notice_the_length_of_its_neighbours():
    """The same short sequences behind a long one and behind padding: equal bits."""
    short = [20, 60, 5, 300, 63]
    blocks, t = [[1600] + short, [-1600] + short], 2048
    q, dout = L.normal((1, t, 2, 64), BF, 1).repeat(2, 1, 1, 1), L.normal((1, t, 2, 64), BF, 4).repeat(2, 1, 1, 1)
    k, v = L.normal((1, t, 1, 64), BF, 2, mean=1.0).repeat(2, 1, 1, 1), L.normal((1, t, 1, 64), BF, 3, mean=8.0, std=0.25).repeat(2, 1, 1, 1)
    got = call(L.positions(t, blocks), q, k, v, dout)
    torch.cuda.synchronize()
    for n in ("out", "dq", "dk", "dv"):
        assert torch.equal(got[n][0, 1600:], got[n][1, 1600:]), n


@pytest.mark.parametrize("causal", [True, False])
def test_long_rows_with_a_distance_bias(causal):
    """They see thousands of keys, and a few have the weight."""
    blocks, t, d = [[2500], [1300, 1200]], 2500, 112
    q, dout = L.normal((2, t, 2, d), BF, 1), L.normal((2, t, 2, d), BF, 4)
    k, v = L.normal((2, t, 1, d), BF, 2, mean=1.0), L.normal((2, t, 1, d), BF, 3, mean=8.0, std=0.25)
    how = dict(causal=causal, window=0, softcap=0.0, slopes=torch.tensor([0.5, 0.1], device=DEV), scale=d ** -0.5)
    got = call(L.positions(t, blocks), q, k, v, dout, **how)
    torch.cuda.synchronize()
    dq, t_dq, _, _, few = expected(blocks, q, k, v, dout, **how)
    assert not bool(few.all())
    L.close(got["dq"], dq, t_dq, "dq")
