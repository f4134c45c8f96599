"""Helpers of the tests of the layers on packed batches: packings by hand and definitions in 64 bits, one sequence at a
time and without any packing, each with a bound on how far a 16- or 32-bit evaluation may be from it.

Bounds: `u` is the rounding error of an element type (half a unit in the last place, relative).  Outputs are rounded once
(u |x|); attention's probabilities and score gradients are rounded to the element type before the second product (u per
term of that sum); sums in 32 bits over n terms err by at most n 2^-24 of the sum of magnitudes."""
import math

import numpy as np
import torch

DEV = "cuda:0"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24, torch.float64: 2.0 ** -53}
E = 2.0 ** -24


def positions(t: int, blocks) -> torch.Tensor:
    """pos [blocks, t] of sequences laid out by their lengths; a negative length is that many padding slots."""
    pos = np.full((len(blocks), t), -1, np.int32)
    for row, here in zip(pos, blocks):
        s = 0
        for n in here:
            if n > 0:
                row[s:s + n] = np.arange(n)
            s += abs(n)
        assert s <= t
    return torch.from_numpy(pos).to(DEV)


def spans(blocks):
    """(block, first slot, end slot) of every sequence."""
    for b, here in enumerate(blocks):
        s = 0
        for n in here:
            if n > 0:
                yield b, s, s + n
            s += abs(n)


def random_blocks(rng, count: int, t: int, mean: float):
    out = []
    for _ in range(count):
        here, room = [], t
        while room > 0:
            n = int(min(room, max(1, rng.geometric(1.0 / mean))))
            if rng.random() < 0.1 and room == n:
                break
            here.append(n)
            room -= n
        out.append(here)
    return out


def normal(shape, dtype, seed, mean=0.0, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(mean, std, generator=g).to(dtype)


def close(got, want, tol, what):
    assert got.shape == want.shape, what
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    if bool(bad.any()):
        i = tuple(int(x) for x in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d outside, first at %s: got %r want %r, off by %.3g, allowed %.3g" % (
            what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(off[i]), float(tol[i])))


def attention(blocks, q, k, v, dout=None, scale=None, softcap=0.0, slopes=None, causal=True, window=0):
    """({name: value}, {name: allowed error}) in float64, from the formulas."""
    dtype = q.dtype
    u, tiny = U[dtype], (2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126)  # below the type's normal range
    nb, t, h, d = q.shape
    hk = k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    z = lambda x, fill=0.0: torch.full(x, fill, dtype=torch.float64, device=q.device)  # noqa: E731
    val = {"out": z(q.shape), "lse": z((nb, h, t), -math.inf)}
    tol = {"out": z(q.shape), "lse": z((nb, h, t))}
    if dout is not None:
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            val[n], tol[n] = z(x.shape), z(x.shape)
    for b, s0, s1 in spans(blocks):
        i = torch.arange(s1 - s0, device=q.device)
        apart = (i[:, None] - i[None, :]).abs()
        ok = torch.ones_like(apart, dtype=torch.bool)
        if causal:
            ok &= i[:, None] >= i[None, :]
        if window:
            ok &= apart < window
        for head in range(h):
            kv = head // (h // hk)
            Q, K, V = q[b, s0:s1, head].double(), k[b, s0:s1, kv].double(), v[b, s0:s1, kv].double()
            raw = scale * (Q @ K.T)
            size = abs(scale) * (Q.abs() @ K.abs().T)
            s, inner = raw, torch.ones_like(raw)
            if softcap:
                th = torch.tanh(raw / softcap)
                s, inner = softcap * th, 1 - th * th
            bias = 0.0 if slopes is None else float(slopes[head]) * apart.double()
            s = (s - bias).masked_fill(~ok, -math.inf)
            lse = torch.logsumexp(s, -1, keepdim=True)
            P = torch.exp(s - lse)
            # a score's error: the product's sum, then a handful of roundings of values up to the score's size
            mag = torch.where(ok, size + (abs(bias) if slopes is not None else 0.0) + softcap, 0.0).amax(-1, keepdim=True)
            e_p = 2 * ((d + 8) * E * torch.where(ok, size, 0.0).amax(-1, keepdim=True) + 16 * E * mag + 16 * E)
            out = P @ V
            n_row = ok.double() @ V.abs()
            t_out = u * out.abs() + (1.05 * u + e_p) * (P @ V.abs()) + tiny * n_row + tiny
            val["out"][b, s0:s1, head], tol["out"][b, s0:s1, head] = out, t_out
            val["lse"][b, head, s0:s1] = lse[:, 0]
            tol["lse"][b, head, s0:s1] = (e_p + 8 * E * (lse.abs() + mag) + 8 * E)[:, 0]
            if dout is None:
                continue
            G = dout[b, s0:s1, head].double()
            dp = G @ V.T
            delta = (G * out).sum(-1, keepdim=True)
            e_delta = (G.abs() * t_out).sum(-1, keepdim=True) + d * E * (G.abs() * out.abs()).sum(-1, keepdim=True)
            ds = P * (dp - delta) * inner
            e_ds = (1.05 * u + 2 * e_p) * ds.abs() + P * (inner * (e_delta + (d + 8) * E * (G.abs() @ V.abs().T)) +
                                                         (dp - delta).abs() * (64 * E + 2 * e_p * (softcap > 0))) + tiny * ok * (1 + (dp - delta).abs())
            val["dq"][b, s0:s1, head] = scale * (ds @ K)
            tol["dq"][b, s0:s1, head] = abs(scale) * (e_ds @ K.abs())
            val["dk"][b, s0:s1, kv] += scale * (ds.T @ Q)
            tol["dk"][b, s0:s1, kv] += abs(scale) * (e_ds.T @ Q.abs())
            val["dv"][b, s0:s1, kv] += P.T @ G
            tol["dv"][b, s0:s1, kv] += ((1.05 * u + 2 * e_p) * P + tiny * ok).T @ G.abs()
    if dout is not None:
        for n in ("dq", "dk", "dv"):
            tol[n] += u * val[n].abs() + tiny
            tol[n] += 64 * E * tol[n] / u  # sums in 32 bits
    return val, tol


def recurrence(blocks, gate, x, dh=None):
    """({name: value}, {name: allowed error}) in float64.  A rounding error e made at a step enters every later state of
    the sequence with weights that sum to at most 1 / (1 - f); with n steps, and n e at most, the smaller of both counts."""
    u = U[x.dtype]
    val = {n: torch.zeros(x.shape, dtype=torch.float64, device=x.device) for n in ("h", "dgate", "dx")}
    tol = {n: torch.zeros_like(val["h"]) for n in ("h", "dgate", "dx")}
    for b, s0, s1 in spans(blocks):
        g, X = gate[b, s0:s1].double(), x[b, s0:s1].double()
        f, keep = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
        n = s1 - s0
        h, mag, err = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(X)
        last, lmag, lerr = X[0] * 0, X[0] * 0, X[0] * 0
        for i in range(n):
            last, lmag = f[i] * last + keep[i] * X[i], f[i] * lmag + keep[i] * X[i].abs()
            lerr = f[i] * lerr + 16 * E * lmag + 8 * E * (1 + g[i].abs()) * (f[i] * lmag + keep[i] * X[i].abs())
            h[i], mag[i], err[i] = last, lmag, lerr
        val["h"][b, s0:s1], tol["h"][b, s0:s1] = h, u * h.abs() + err + 1e-37
        if dh is None:
            continue
        D = dh[b, s0:s1].double()
        G, gmag, gerr = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(X)
        last, lmag, lerr = X[0] * 0, X[0] * 0, X[0] * 0
        for i in range(n - 1, -1, -1):
            last, lmag = D[i] + last, D[i].abs() + lmag
            lerr = lerr + 16 * E * lmag
            G[i], gmag[i], gerr[i] = last, lmag, lerr
            last, lmag, lerr = f[i] * last, f[i] * lmag, f[i] * (lerr + 8 * E * (1 + g[i].abs()) * lmag)
        before, bmag, berr = torch.zeros_like(X), torch.zeros_like(X), torch.zeros_like(X)
        before[1:], bmag[1:], berr[1:] = h[:-1], mag[:-1], err[:-1]
        rel = 16 * E * (1 + g.abs())
        val["dx"][b, s0:s1] = keep * G
        tol["dx"][b, s0:s1] = u * (keep * G).abs() + keep * (gerr + rel * gmag) + 1e-37
        dg = G * (before - X) * f * keep
        val["dgate"][b, s0:s1] = dg
        tol["dgate"][b, s0:s1] = u * dg.abs() + f * keep * ((gerr + rel * gmag) * (before - X).abs() +
                                                         G.abs() * (berr + 16 * E * (bmag + X.abs()))) + 1e-37
    if x.dtype == torch.float16:
        for n in tol:
            tol[n] += 2.0 ** -25  # below its normal range
    return val, tol
