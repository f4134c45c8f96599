"""Definitions in 64 bits of layer norm, the short convolution and the state-space scan, one sequence at a time and without any
packing, each with a bound on how far an evaluation in 32 bits with one rounding at the end may be from it.

Bounds: E = 2^-24 is half a unit of a 32-bit number, U[dtype] of an output's type.  A sum of n terms errs by at most n E of the sum
of magnitudes, in any order; an exponential, a reciprocal or a product in hardware by a few E of itself, an exponential also by what
its argument errs.  Errors are carried along with the values: err(f(x)) <= |f'| err(x) + rounding."""
import torch

import layer_util as L

E, U, spans = L.E, L.U, L.spans


def zeros(shape):
    return torch.zeros(shape, dtype=torch.float64, device=L.DEV)


def rounded(val, tol, dtype):
    """the tolerance with the output's own rounding; in fp16 half a step of the smallest numbers"""
    return tol + U[dtype] * val.abs() + (2.0 ** -25 if dtype == torch.float16 else 1e-37)


def norm(blocks, x, weight, bias, eps, dy=None):
    c = x.shape[-1]
    w = torch.ones(c, device=L.DEV).double() if weight is None else weight.double()
    b = torch.zeros(c, device=L.DEV).double() if bias is None else bias.double()
    val = {n: zeros(x.shape) for n in ("y", "dx")} | {n: zeros((c,)) for n in ("dweight", "dbias")} | {"stats": zeros((*x.shape[:2], 2))}
    tol = {n: torch.zeros_like(v) for n, v in val.items()}
    k = 64 * E  # a sum over the channels: at most 32 in a thread, 5 exchanges, 16 warps, and a product
    frames = 0
    for q, s0, s1 in spans(blocks):
        X = x[q, s0:s1].double()
        frames += s1 - s0
        m = X.mean(-1, keepdim=True)
        r = 1 / torch.sqrt((X - m).square().mean(-1, keepdim=True) + eps)
        n = (X - m) * r
        e_m = k * X.abs().mean(-1, keepdim=True) + E * m.abs()
        e_r = k * r + r ** 3 * e_m.square()
        e_n = r * (e_m + 2 * E * (X - m).abs()) + e_r * (X - m).abs() + 2 * E * n.abs()
        y = n * w + b
        val["y"][q, s0:s1], tol["y"][q, s0:s1] = y, rounded(y, w.abs() * e_n + 4 * E * ((n * w).abs() + b.abs()), x.dtype)
        val["stats"][q, s0:s1], tol["stats"][q, s0:s1] = torch.cat((m, r), -1), torch.cat((e_m, e_r + E * r), -1)
        if dy is None:
            continue
        D = dy[q, s0:s1].double()
        g = D * w
        m1, m2 = g.mean(-1, keepdim=True), (g * n).mean(-1, keepdim=True)
        e1 = k * g.abs().mean(-1, keepdim=True)
        e2 = k * (g * n).abs().mean(-1, keepdim=True) + (g.abs() * e_n).mean(-1, keepdim=True)
        inner = g - m1 - n * m2
        dx = r * inner
        e = r * (e1 + n.abs() * e2 + e_n * m2.abs() + 4 * E * (g.abs() + m1.abs() + (n * m2).abs())) + e_r * inner.abs() + 4 * E * dx.abs()
        val["dx"][q, s0:s1], tol["dx"][q, s0:s1] = dx, rounded(dx, e, x.dtype)
        val["dweight"] += (D * n).sum(0)
        val["dbias"] += D.sum(0)
        # (the last factors count the additions, at most one per frame and CTA)
        tol["dweight"] += (D.abs() * e_n).sum(0) + (x.shape[0] * x.shape[1] + 64) * E * (D * n).abs().sum(0) + 1e-37
        tol["dbias"] += (x.shape[0] * x.shape[1] + 64) * E * D.abs().sum(0) + 1e-37
    return val, tol


def silu(u, e_u):
    """(sigmoid, value, its error, slope, its error) at u, which errs by e_u; |slope| <= 1.1, |slope'| <= 0.5"""
    s = 1 / (1 + torch.exp(-u))
    rel = (8 + 4 * u.abs()) * E
    slope = s * (1 + u * (1 - s))
    return s, u * s, 1.1 * e_u + (u * s).abs() * rel, slope, 0.5 * e_u + (8 + 4 * u.abs()) * E * (s + (u * s).abs()) + 4 * E


def conv(blocks, x, weight, bias, act, dy=None):
    c, taps = weight.shape
    w = weight.double()
    b = zeros((c,)) if bias is None else bias.double()
    val = {n: zeros(x.shape) for n in ("y", "dx")} | {"dweight": zeros((c, taps)), "dbias": zeros((c,))}
    tol = {n: torch.zeros_like(v) for n, v in val.items()}
    tails = []
    for q, s0, s1 in spans(blocks):
        X = torch.cat((zeros((taps - 1, c)), x[q, s0:s1].double()))
        n = s1 - s0
        tails.append(X[n:] if taps > 1 else X[:0])
        seen = torch.stack([X[i:i + n] for i in range(taps)], -1)  # [n, c, taps], the frame itself last
        u = (seen * w).sum(-1) + b
        e_u = (taps + 2) * E * ((seen * w).abs().sum(-1) + b.abs())
        slope, e_slope = torch.ones_like(u), torch.zeros_like(u)
        y, e_y = u, e_u
        if act:
            _, y, e_y, slope, e_slope = silu(u, e_u)
        val["y"][q, s0:s1], tol["y"][q, s0:s1] = y, rounded(y, e_y, x.dtype)
        if dy is None:
            continue
        D = dy[q, s0:s1].double()
        du, e_du = D * slope, D.abs() * e_slope + 2 * E * (D * slope).abs()
        dX, e_X = torch.zeros_like(X), torch.zeros_like(X)
        for i in range(taps):
            dX[i:i + n] += w[:, i] * du
            e_X[i:i + n] += w[:, i].abs() * (e_du + (taps + 2) * E * du.abs())
            val["dweight"][:, i] += (du * seen[..., i]).sum(0)
            tol["dweight"][:, i] += (e_du * seen[..., i].abs() + (x.shape[0] * x.shape[1] + 64) * E * (du * seen[..., i]).abs()).sum(0) + 1e-37
        val["dx"][q, s0:s1], tol["dx"][q, s0:s1] = dX[taps - 1:], rounded(dX[taps - 1:], e_X[taps - 1:], x.dtype)
        val["dbias"] += du.sum(0)
        tol["dbias"] += (e_du + (x.shape[0] * x.shape[1] + 64) * E * du.abs()).sum(0) + 1e-37
    return val, tol, tails


def delta(raw, softplus):
    """(value, its error, slope, its error) of softplus or of the identity, at a sum rounded to 32 bits"""
    if not softplus:
        return raw, E * raw.abs(), torch.ones_like(raw), torch.zeros_like(raw)
    s = 1 / (1 + torch.exp(-raw))
    d = torch.logaddexp(raw, torch.zeros_like(raw))
    return d, 16 * E * d + 2 * E * raw.abs() * s, s, 16 * E * s + 2 * E * raw.abs() * s


def scan(blocks, x, dt, a, b, c, d=None, dt_bias=None, z=None, softplus=True, dy=None, start=None, ends=None):
    """Values and tolerances of all outputs; "last": the states behind the sequences, in the order of spans().  start: [sequences,
    channels, states], states to begin with."""
    dtype, (ch, n) = x.dtype, a.shape
    A = a.double()
    D = zeros((ch,)) if d is None else d.double()
    names = ("y", "dx", "ddt") + (("dz",) if z is not None else ())
    val = {k: zeros(x.shape) for k in names} | {k: zeros(b.shape) for k in ("db", "dc")} | {"da": zeros((ch, n))} | {k: zeros((ch,)) for k in ("dd", "ddt_bias")}
    tol = {k: torch.zeros_like(v) for k, v in val.items()}
    last, last_tol = [], []
    frames = x.shape[0] * x.shape[1] + 64
    for i, (q, s0, s1) in enumerate(spans(blocks)):
        X, B, C = (y[q, s0:s1].double() for y in (x, b, c))
        raw = dt[q, s0:s1].double() + (0 if dt_bias is None else dt_bias.double())
        dl, e_dl, slope, e_slope = delta(raw, softplus)
        u, e_u = dl * X, X.abs() * e_dl + 2 * E * (dl * X).abs()
        k = s1 - s0
        decay = torch.exp(dl[..., None] * A)
        e_decay = decay * (A.abs() * e_dl[..., None] + 4 * E * (dl[..., None] * A).abs() + 4 * E)
        push = u[..., None] * B[:, None]
        H, eH, W, eW = (zeros((k, ch, n)) for _ in range(4))
        h = zeros((ch, n)) if start is None else start[i].double()
        eh = torch.zeros_like(h)
        for s in range(k):
            if s or start is not None:
                W[s], eW[s] = decay[s] * h, decay[s] * eh + e_decay[s] * (h.abs() + eh) + 2 * E * (decay[s] * h).abs()
            h = W[s] + push[s]
            eh = eW[s] + B[s].abs() * e_u[s][:, None] + 2 * E * (push[s].abs() + h.abs())
            H[s], eH[s] = h, eh
        last.append(h)
        last_tol.append(eh + 1e-37)
        v = (H * C[:, None]).sum(-1) + D * X
        e_v = (C[:, None].abs() * eH).sum(-1) + (n + 8) * E * (H * C[:, None]).abs().sum(-1) + 4 * E * (D * X).abs()
        gate, e_gate = torch.ones_like(v), torch.zeros_like(v)
        if z is not None:
            _, gate, e_gate, z_slope, e_z_slope = silu(z[q, s0:s1].double(), 0.0)
        y = v * gate
        val["y"][q, s0:s1], tol["y"][q, s0:s1] = y, rounded(y, gate.abs() * e_v + v.abs() * e_gate + 4 * E * y.abs(), dtype)
        if dy is None:
            continue
        G0 = dy[q, s0:s1].double()
        dv, e_dv = G0 * gate, G0.abs() * e_gate + 4 * E * (G0 * gate).abs()
        if z is not None:
            dz = G0 * v * z_slope
            val["dz"][q, s0:s1] = dz
            tol["dz"][q, s0:s1] = rounded(dz, G0.abs() * (e_v * z_slope.abs() + v.abs() * e_z_slope) + 4 * E * dz.abs(), dtype)
        G, eG = zeros((k, ch, n)), zeros((k, ch, n))
        e, ee = zeros((ch, n)), zeros((ch, n))
        for s in range(k - 1, -1, -1):
            part = dv[s][:, None] * C[s]
            g = part + e
            eg = C[s].abs() * e_dv[s][:, None] + ee + 2 * E * (part.abs() + g.abs())
            G[s], eG[s] = g, eg
            e, ee = decay[s] * g, decay[s] * eg + e_decay[s] * (g.abs() + eg) + 2 * E * (decay[s] * g).abs()
        dc, db = (dv[..., None] * H).sum(1), (u[..., None] * G).sum(1)
        e_dc = (dv.abs()[..., None] * eH + e_dv[..., None] * H.abs()).sum(1) + (ch + 8) * E * (dv[..., None] * H).abs().sum(1)
        e_db = (u.abs()[..., None] * eG + e_u[..., None] * G.abs()).sum(1) + (ch + 8) * E * (u[..., None] * G).abs().sum(1)
        val["db"][q, s0:s1], tol["db"][q, s0:s1] = db, rounded(db, e_db, dtype)
        val["dc"][q, s0:s1], tol["dc"][q, s0:s1] = dc, rounded(dc, e_dc, dtype)
        sb, sa = (G * B[:, None]).sum(-1), (G * W * A).sum(-1)
        e_sb = (eG * B[:, None].abs()).sum(-1) + (n + 8) * E * (G * B[:, None]).abs().sum(-1)
        e_gw = G.abs() * eW + eG * W.abs() + 2 * E * (G * W).abs()
        e_sa = (e_gw * A.abs()).sum(-1) + (n + 8) * E * (G * W * A).abs().sum(-1)
        val["da"] += (G * W * dl[..., None]).sum(0)
        tol["da"] += (e_gw * dl[..., None].abs() + (G * W).abs() * e_dl[..., None] + frames * E * (G * W * dl[..., None]).abs()).sum(0) + 1e-37
        dx = dl * sb + D * dv
        e_dx = dl.abs() * e_sb + e_dl * sb.abs() + D.abs() * e_dv + 4 * E * ((dl * sb).abs() + (D * dv).abs())
        val["dx"][q, s0:s1], tol["dx"][q, s0:s1] = dx, rounded(dx, e_dx, dtype)
        inner = X * sb + sa
        e_inner = X.abs() * e_sb + e_sa + 4 * E * ((X * sb).abs() + sa.abs())
        ddt, e_ddt = inner * slope, slope * e_inner + inner.abs() * e_slope + 4 * E * (inner * slope).abs()
        val["ddt"][q, s0:s1], tol["ddt"][q, s0:s1] = ddt, rounded(ddt, e_ddt, dtype)
        val["ddt_bias"] += ddt.sum(0)
        tol["ddt_bias"] += (e_ddt + frames * E * ddt.abs()).sum(0) + 1e-37
        val["dd"] += (dv * X).sum(0)
        tol["dd"] += (e_dv * X.abs() + frames * E * (dv * X).abs()).sum(0) + 1e-37
    val["last"] = torch.stack(last) if last else zeros((0, ch, n))
    tol["last"] = torch.stack(last_tol) if last else zeros((0, ch, n))
    return val, tol


def scan_inputs(b, t, ch, n, dtype, seed, z=True):
    """What a layer has: x, dt, b, c, z, dy of the type; a, d, dt_bias in 32 bits, delta between 0.001 and 0.3."""
    g = torch.Generator(device=L.DEV)
    g.manual_seed(seed)
    f32 = torch.float32

    def make(*shape, std=1.0, mean=0.0, dt=dtype):
        return torch.empty(shape, dtype=f32, device=L.DEV).normal_(mean, std, generator=g).to(dt)

    i = {"x": make(b, t, ch), "dt": make(b, t, ch, std=0.8), "b": make(b, t, n), "c": make(b, t, n), "dy": make(b, t, ch),
         "z": make(b, t, ch) if z else None, "a": -make(ch, n, std=0.7, dt=f32).exp() * torch.arange(1, n + 1, device=L.DEV),
         "d": make(ch, mean=1.0, std=0.3, dt=f32), "dt_bias": make(ch, mean=-4.0, dt=f32)}
    return i


def sequence_numbers(pos, shuffle=None):
    """(seq_id [blocks, t], how many); shuffle: a permutation that gives sequence k of spans() the number shuffle[k]"""
    starts = (pos == 0).int().cumsum(1).int() - 1
    per = (pos == 0).sum(1)
    first = per.cumsum(0) - per
    ids = torch.where(pos >= 0, starts + first[:, None].int(), -1)
    if shuffle is not None:
        ids = torch.where(pos >= 0, shuffle.to(torch.int32)[ids.clamp(min=0).long()], -1)
    return ids.to(torch.int32).contiguous(), int(per.sum())
