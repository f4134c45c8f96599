"""Attention in fp16 where its range is short: weights and score gradients far below its smallest normal number, and far above
its largest, inside a computation whose inputs and outputs it holds.

Bound: as in layer_util, but no term may be lost: P is rounded to u = 2^-11 of itself or 2^-38 (2^-31 of the row's largest in the forward
pass).  A dS is rounded to u of itself, or 2^-34 of the product of the largest of the first eight elements of dout and of v at its row's own slot (the
query's for dq, the key's for dk, there with the first of the heads that share it), or 2^-39 of the row's largest dS where that is larger."""
import math

import pytest
import torch

import layer_util as L
from test_gpu_attention import FP, call

pytestmark = pytest.mark.gpu
DEV, E, U = L.DEV, L.E, L.U[FP]


def expected(blocks, q, k, v, dout, causal):
    """({name: value}, {name: allowed error}) in float64."""
    nb, t, h, d = q.shape
    scale = d ** -0.5
    val = {n: torch.zeros(x.shape, dtype=torch.float64, device=DEV) for n, x in (("out", q), ("dq", q), ("dk", k), ("dv", v))}
    tol = {n: torch.zeros_like(x) for n, x in val.items()}
    for b, s0, s1 in L.spans(blocks):
        n = s1 - s0
        i = torch.arange(n, device=DEV)
        ok = i[:, None] >= i[None, :] if causal else torch.ones((n, n), dtype=torch.bool, device=DEV)
        for head in range(h):
            kv = head // (h // k.shape[2])
            Q, K, V, G = (x.double() for x in (q[b, s0:s1, head], k[b, s0:s1, kv], v[b, s0:s1, kv], dout[b, s0:s1, head]))
            size = torch.where(ok, scale * (Q.abs() @ K.abs().T), 0.0).amax(-1, keepdim=True)
            P = torch.softmax((scale * (Q @ K.T)).masked_fill(~ok, -math.inf), -1)
            e_p = 2 * ((d + 8) * E * size + 16 * E * size + 16 * E)  # relative
            r_p = (1.05 * U + e_p + n * E) * P  # rounded as an operand; sums in 32 bits
            out, dP = P @ V, G @ V.T
            t_out = U * out.abs() + (r_p + 2.0 ** -31 * P.amax(-1, keepdim=True) * ok) @ V.abs() + 2.0 ** -25
            delta = (P * dP).sum(-1, keepdim=True)
            e_delta = (G.abs() * t_out).sum(-1, keepdim=True) + d * E * (G.abs() * out.abs()).sum(-1, keepdim=True)
            dS = P * (dP - delta)
            e_ds = (1.05 * U + 2 * e_p + n * E) * dS.abs() + P * (e_delta + (d + 8) * E * (G.abs() @ V.abs().T))
            top = dS.abs() + e_ds
            V8 = V[:, :8].abs().amax(-1)
            own_q, own_k = G[:, :8].abs().amax(-1) * V8, dout[b, s0:s1, kv * (h // k.shape[2]), :8].double().abs().amax(-1) * V8
            q_step = torch.maximum(2.0 ** -34 * own_q, 2.0 ** -39 * top.amax(1))[:, None] * ok
            k_step = torch.maximum(2.0 ** -34 * own_k, 2.0 ** -39 * top.amax(0))[None, :] * ok
            at = lambda x, y: val[x].__setitem__((b, slice(s0, s1), y[0]), val[x][b, s0:s1, y[0]] + y[1])  # noqa: E731
            add = lambda x, y: tol[x].__setitem__((b, slice(s0, s1), y[0]), tol[x][b, s0:s1, y[0]] + y[1])  # noqa: E731
            at("out", (head, out)), add("out", (head, t_out))
            at("dq", (head, scale * (dS @ K))), add("dq", (head, scale * ((e_ds + q_step) @ K.abs())))
            at("dk", (kv, scale * (dS.T @ Q))), add("dk", (kv, scale * ((e_ds + k_step).T @ Q.abs())))
            at("dv", (kv, P.T @ G)), add("dv", (kv, (r_p + 2.0 ** -38 * ok).T @ G.abs()))
    for n in ("dq", "dk", "dv"):
        tol[n] += U * val[n].abs() + 2.0 ** -25
        tol[n] += 64 * E * tol[n] / U
    return val, tol


def compare(blocks, t, q, k, v, dout, causal):
    got = call(L.positions(t, blocks), q, k, v, dout, causal=causal)
    torch.cuda.synchronize()
    val, tol = expected(blocks, q, k, v, dout, causal)
    for n in val:
        assert float(val[n].abs().max()) < 65000  # the type holds the result
        L.close(got[n], val[n], tol[n], n)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [1e-2, 1e-4])
@pytest.mark.parametrize("causal", [True, False])
def test_small_gradients_over_many_keys(causal, size, d):
    """Score gradients of 1e-6 and less.  Keys and queries share a direction, so what is lost of them adds up."""
    blocks, t = [[4000, 90], [30, 2000, -60, 2000]], 4090
    q, k = L.normal((2, t, 2, d), FP, 1, mean=0.3, std=0.2), L.normal((2, t, 1, d), FP, 2, mean=0.5, std=0.3)
    v, dout = L.normal((2, t, 1, d), FP, 3), L.normal((2, t, 2, d), FP, 4, std=size)
    compare(blocks, t, q, k, v, dout, causal)


@pytest.mark.parametrize("d", [40, 96])
@pytest.mark.parametrize("causal", [True, False])
def test_score_gradients_above_the_largest_number(causal, d):
    """dS of 1e5 and more between operands and results that fp16 holds."""
    blocks, t = [[8, 3, 200, 1, 2], [214]], 214
    q, k = L.normal((2, t, 2, d), FP, 1, std=0.02), L.normal((2, t, 1, d), FP, 2, std=0.02)
    v, dout = L.normal((2, t, 1, d), FP, 3, std=100.0), L.normal((2, t, 2, d), FP, 4, std=1000.0)
    compare(blocks, t, q, k, v, dout, causal)


@pytest.mark.parametrize("causal", [True, False])
def test_gradients_of_all_sizes_side_by_side(causal):
    """dout from 1e-6 to 1e3 from one query to the next, and from one sequence to the next; growing along a third."""
    blocks, t, d = [[700, 500, 300]], 1500, 64
    q, k, v = L.normal((1, t, 2, d), FP, 1), L.normal((1, t, 1, d), FP, 2), L.normal((1, t, 1, d), FP, 3)
    g = torch.Generator(device=DEV).manual_seed(5)
    size = 10.0 ** (torch.rand((t,), generator=g, device=DEV) * 9 - 6)
    size[700:1200] = 1e-5
    size[1200:] = 10.0 ** torch.linspace(-6, 3, 300, device=DEV)
    dout = (L.normal((1, t, 2, d), torch.float32, 4) * size[None, :, None, None]).to(FP)
    compare(blocks, t, q, k, v, dout, causal)


def test_weights_far_below_one():
    """Keys whose weights are 1e-6 and less everywhere: their dv is small, and not lost."""
    blocks, t, d = [[3000]], 3000, 64
    q, k = L.normal((1, t, 1, d), FP, 1, std=0.1), L.normal((1, t, 1, d), FP, 2, std=0.1)
    q[..., 0], k[..., 0] = 8.0, 0.0
    k[:, ::3, :, 0] = -9.0  # scores 9 below the others'
    v, dout = L.normal((1, t, 1, d), FP, 3), L.normal((1, t, 1, d), FP, 4, mean=2.0)
    compare(blocks, t, q, k, v, dout, False)


@pytest.mark.parametrize("d", [64, 128])
def test_gradients_that_come_from_other_slots_only(d):
    """dout is zero but for the last queries of a sequence, so that nothing of a row's own slot tells how large its dS are: they would not
    fit what that suggests.  The sequences beside it, in the same 128 rows, keep their bits."""
    blocks, t = [[60, 900, 64], [900, 60, 64]], 1024
    pos = L.positions(t, blocks)
    q, k, v, dout = (L.normal((2, t, n, d), FP, i) for n, i in ((2, 1), (1, 2), (1, 3), (2, 4)))
    plain = {n: x.clone() for n, x in call(pos, q, k, v, dout).items()}
    spans = [(60, 960), (0, 900)]
    for b, (s0, s1) in enumerate(spans):
        dout[b, s0:s1 - 5] = 0.0
    got = call(pos, q, k, v, dout)
    torch.cuda.synchronize()
    val, tol = expected(blocks, q, k, v, dout, True)
    for n in val:
        L.close(got[n], val[n], tol[n], n)
    for b, (s0, s1) in enumerate(spans):
        for n in ("dq", "dk", "dv"):
            assert torch.equal(got[n][b, :s0], plain[n][b, :s0]) and torch.equal(got[n][b, s1:], plain[n][b, s1:]), n
