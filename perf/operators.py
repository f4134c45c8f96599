"""Cases for the sequence-mixing operators that read a packed batch's positions: rotary positions, attention inside
the sequences of a block, and a gated linear recurrence that restarts with every sequence.

A packed batch holds several sequences in each block of `t` slots; `pos[b, s]` is a slot's position in its sequence and
-1 on padding, as bload_pack writes it.  Every operator works inside sequences only:

  rotary      y = factor * R(pos) x on the first 2 * len(inv_freq) elements of every head; padding is copied.
  attention   score = scale * q.k, optionally cap * tanh(score / cap), optionally - slope[head] * |i - j|; softmax over
              the slots j of i's sequence (j <= i when causal, |i - j| < window when given); padding gives 0.
  recurrence  f = sigmoid(gate), h = f * h_prev + (1 - f) * x, h_prev = 0 at a sequence's start; padding gives 0.

`own` selects between the framework's calls and plain torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # Toy clips (blocks of 64 slots): one batch is a handful of kilobytes, so this is the latency of a call.
        {"name": "rotary toy", "op": "rotary", "grad": False, "b": 8, "t": 64, "h": 16, "d": 64, "rot": 64,
         "interleaved": False, "factor": 1.0, "base": 10000.0, "dtype": "fp16", "docs": "toy"},
        # Token blocks: the 16 query and 4 key heads of a fused projection, all of the head rotated, half layout.
        {"name": "rotary tokens", "op": "rotary", "grad": False, "b": 16, "t": 4096, "h": 20, "d": 128, "rot": 128,
         "interleaved": False, "factor": 1.0, "base": 10000.0, "dtype": "bf16", "docs": "tokens"},
        # Gradient of interleaved positions on part of the head, stretched for long contexts (factor and base), 32 bits.
        {"name": "rotary grad partial", "op": "rotary", "grad": True, "b": 16, "t": 1000, "h": 16, "d": 80, "rot": 32,
         "interleaved": True, "factor": 1.2079, "base": 500000.0, "dtype": "fp32", "docs": "features"},
        # One batch of toy clips through a small layer: latency.
        {"name": "recurrence toy", "op": "recurrence", "train": False, "b": 8, "t": 64, "d": 512, "dtype": "bf16",
         "docs": "toy"},
        # Forward pass over per-frame features (16 blocks of 1000 frames, 1024 channels), validation.
        {"name": "recurrence features", "op": "recurrence", "train": False, "b": 16, "t": 1000, "d": 1024,
         "dtype": "fp16", "docs": "features"},
        # Training step of the heavy-tailed workload: 8 blocks of 10,000 frames, 2048 channels.
        {"name": "recurrence train heavy", "op": "recurrence", "train": True, "b": 8, "t": 10000, "d": 2048,
         "dtype": "bf16", "docs": "heavy"},
        # One long sequence, few and odd channels, 32 bits: the time axis is all there is to split.
        {"name": "recurrence train long", "op": "recurrence", "train": True, "b": 1, "t": 30001, "d": 251,
         "dtype": "fp32", "docs": "single"},
        # Toy clips, causal: latency.
        {"name": "attention toy", "op": "attention", "train": False, "b": 8, "t": 64, "h": 8, "hkv": 8, "d": 64,
         "causal": True, "window": 0, "cap": 0.0, "slopes": False, "dtype": "fp16", "docs": "toy"},
        # Video features attend in both directions inside a clip: 16 blocks of 1000 frames.
        {"name": "attention features", "op": "attention", "train": False, "b": 16, "t": 1000, "h": 16, "hkv": 16,
         "d": 64, "causal": False, "window": 0, "cap": 0.0, "slopes": False, "dtype": "fp16", "docs": "features"},
        # Training step on token blocks: causal, grouped key heads.
        {"name": "attention train tokens", "op": "attention", "train": True, "b": 4, "t": 4096, "h": 16, "hkv": 4,
         "d": 128, "causal": True, "window": 0, "cap": 0.0, "slopes": False, "dtype": "bf16", "docs": "tokens"},
        # Training step on heavy-tailed blocks with capped scores and a bias that grows with distance, odd head size.
        {"name": "attention train capped", "op": "attention", "train": True, "b": 2, "t": 5003, "h": 8, "hkv": 4,
         "d": 88, "causal": True, "window": 0, "cap": 30.0, "slopes": True, "dtype": "bf16", "docs": "heavy"},
        # Training step on one long sequence that fills its block: bound by the matrix products.
        {"name": "attention train long", "op": "attention", "train": True, "b": 1, "t": 16384, "h": 4, "hkv": 2,
         "d": 128, "causal": True, "window": 0, "cap": 0.0, "slopes": False, "dtype": "bf16", "docs": "single"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "recurrence", "attention", "attention"])
    docs = rng.choice(["toy", "features", "tokens", "heavy", "single"])
    if op == "rotary":
        d = 8 * rng.randint(1, 16)
        t = _log_int(rng, 1, 16384)
        rows = _log_int(rng, 1, max(1, 16 * 4096 * 20 * 128 // (t * d * 2)))  # blocks x heads, at most half the largest case in 32 bits
        h = min(rows, rng.randint(1, 32))
        return {"op": op, "grad": rng.random() < 0.5, "b": max(1, rows // h), "t": t, "h": h, "d": d,
                "rot": min(d, 2 * rng.randint(1, max(1, d // 2))), "interleaved": rng.random() < 0.5,
                "factor": rng.choice([1.0, 1.1386]), "base": rng.choice([10000.0, 500000.0]),
                "dtype": rng.choice(["fp32", "fp16", "bf16"]), "docs": docs}
    if op == "recurrence":
        t = _log_int(rng, 1, 32768)
        d = _log_int(rng, 1, 4096)
        if rng.random() < 0.7:
            d = -(-d // 8) * 8
        b = _log_int(rng, 1, max(1, min(64, 8 * 10000 * 2048 // (2 * t * d))))
        return {"op": op, "train": rng.random() < 0.6, "b": b, "t": t, "d": d,
                "dtype": rng.choice(["fp32", "fp16", "bf16"]), "docs": docs}
    t = _log_int(rng, 1, 16000)
    rows = _log_int(rng, 1, max(1, min(512, 4 * 16384 * 16384 // (t * t))))  # blocks x heads
    hkv = min(rows, rng.choice([1, 2, 4, 8]))
    g = min(rows // hkv, rng.choice([1, 2, 4]))
    causal = rng.random() < 0.7
    return {"op": op, "train": rng.random() < 0.6, "b": max(1, rows // (hkv * g)), "t": t, "h": hkv * g, "hkv": hkv,
            "d": rng.choice([64, 128, 8 * rng.randint(2, 16)]), "causal": causal,
            "window": rng.choice([0, 0, rng.randint(1, 2048)]), "cap": rng.choice([0.0, 0.0, 30.0, 50.0]),
            "slopes": rng.random() < 0.3, "dtype": rng.choice(["fp16", "bf16"]), "docs": docs}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _lengths(docs, t, n, rng):
    """n sequence lengths of one of the framework's workloads, at most t."""
    if docs == "toy":
        x = rng.integers(2, 65, n)
    elif docs == "features":
        x = np.rint(rng.lognormal(math.log(30.0), 1.0, n))
    elif docs == "tokens":
        x = np.clip(rng.zipf(1.2, n), 8, 4096)
    elif docs == "heavy":
        x = np.floor(20.0 * (1.0 + rng.pareto(1.5, n)))
    else:
        x = np.full(n, t)
    return np.clip(x, 1, t).astype(np.int64)


def _blocks(case, seed):
    """The sequence lengths of each block: drawn at random while one fits, the rest of the block is padding."""
    rng = np.random.default_rng(seed)
    out = []
    for _ in range(case["b"]):
        room, here, misses = case["t"], [], 0
        while room > 0 and misses < 2:
            for x in _lengths(case["docs"], case["t"], 64, rng).tolist():
                if x <= room:
                    here.append(x)
                    room -= x
                    misses = 0
            misses += 1
        out.append(here)
    return out


def _positions(case, blocks):
    pos = np.full((case["b"], case["t"]), -1, np.int32)
    for row, here in zip(pos, blocks):
        s = 0
        for n in here:
            row[s:s + n] = np.arange(n, dtype=np.int32)
            s += n
    return pos



def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dt = TYPES[case["dtype"]]
    b, t, d = case["b"], case["t"], case["d"]
    state = {"case": dict(case), "pos": torch.from_numpy(_positions(case, _blocks(case, seed))).to(dev)}

    def normal(*shape, mean=0.0, std=1.0):
        return torch.empty(shape, dtype=torch.float32, device=dev).normal_(mean, std, generator=g).to(dt)

    if case["op"] == "rotary":
        i = torch.arange(case["rot"] // 2, dtype=torch.float64)
        state["inv_freq"] = (case["base"] ** (-2.0 * i / case["rot"])).float().to(dev)
        state["x"] = normal(b, t, case["h"], d)
        state["y"] = torch.empty_like(state["x"])
    elif case["op"] == "recurrence":
        state["gate"], state["x"] = normal(b, t, d, mean=3.0, std=1.5), normal(b, t, d)
        if case["train"]:
            state["dh"] = normal(b, t, d)
        state["h"] = torch.empty_like(state["x"])
        state["dgate"], state["dx"] = torch.empty_like(state["x"]), torch.empty_like(state["x"])
    else:
        h, hkv = case["h"], case["hkv"]
        state["q"], state["k"], state["v"] = normal(b, t, h, d, std=1.5), normal(b, t, hkv, d), normal(b, t, hkv, d)
        if case["train"]:
            state["dout"] = normal(b, t, h, d)
        state["slopes"] = torch.tensor([2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device=dev) if case["slopes"] else None
        state["out"] = torch.empty_like(state["q"])
        state["lse"] = torch.empty((b, h, t), dtype=torch.float32, device=dev)
        state["delta"] = torch.empty((b, h, t), dtype=torch.float32, device=dev)
        state["dq"], state["dk"], state["dv"] = (torch.empty_like(state[n]) for n in ("q", "k", "v"))
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["op"]](case, state)


def _own_rotary(c, s):
    import paper_2310_10879_b200 as B
    call = B.bload_rotary_grad if c["grad"] else B.bload_rotary
    call(s["pos"], s["x"], s["y"], s["inv_freq"], interleaved=c["interleaved"], factor=c["factor"])
    return {"y": s["y"]}


def _own_recurrence(c, s):
    import paper_2310_10879_b200 as B
    carry, work = B.bload_recurrence_buffers(s["pos"], s["x"])  # states kept for the backward pass, and scratch
    B.bload_recurrence(s["pos"], s["gate"], s["x"], s["h"], carry, work)
    if not c["train"]:
        return {"h": s["h"]}
    B.bload_recurrence_grad(s["pos"], s["gate"], s["x"], carry, s["dh"], s["dgate"], s["dx"], work)
    return {"h": s["h"], "dgate": s["dgate"], "dx": s["dx"]}


def _own_attention(c, s):
    import paper_2310_10879_b200 as B
    how = {"softcap": c["cap"], "slopes": s["slopes"], "causal": c["causal"], "window": c["window"]}
    B.bload_attention(s["pos"], s["q"], s["k"], s["v"], s["out"], s["lse"], **how)
    if not c["train"]:
        return {"out": s["out"], "lse": s["lse"]}
    B.bload_attention_grad(s["pos"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"],
                           s["delta"], **how)
    return {"out": s["out"], "lse": s["lse"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}


def _plain_rotary(c, s):
    x, n = s["x"].float(), c["rot"] // 2
    pos = s["pos"]
    angle = pos[..., None].float() * s["inv_freq"]
    cos, sin = angle.cos()[:, :, None] * c["factor"], angle.sin()[:, :, None] * c["factor"]
    if c["grad"]:
        sin = -sin
    if c["interleaved"]:
        u, w = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        y = torch.stack((u * cos - w * sin, w * cos + u * sin), -1).flatten(-2)
    else:
        u, w = x[..., :n], x[..., n:2 * n]
        y = torch.cat((u * cos - w * sin, w * cos + u * sin), -1)
    y = torch.cat((y, x[..., 2 * n:]), -1)
    return {"y": torch.where((pos >= 0)[..., None, None], y, x).to(s["x"].dtype)}


def _linear_scan(a, u):
    """h[s] = a[s] * h[s - 1] + u[s] along dim 1, by doubling the reach of every slot."""
    k = 1
    while k < a.shape[1]:
        u = torch.cat((u[:, :k], u[:, k:] + a[:, k:] * u[:, :-k]), 1)
        a = torch.cat((a[:, :k], a[:, k:] * a[:, :-k]), 1)
        k *= 2
    return u


def _plain_recurrence(c, s):
    pos = s["pos"][..., None]
    gate, x = s["gate"].float(), s["x"].float()
    f, keep = torch.sigmoid(gate), torch.sigmoid(-gate)
    a = torch.where(pos > 0, f, 0.0)
    h = _linear_scan(a, torch.where(pos >= 0, keep * x, 0.0))
    out = {"h": h.to(s["x"].dtype)}
    if c["train"]:
        a_next = torch.cat((a[:, 1:], torch.zeros_like(a[:, :1])), 1)
        dh = torch.where(pos >= 0, s["dh"].float(), 0.0)
        g = _linear_scan(a_next.flip(1), dh.flip(1)).flip(1)
        h_prev = torch.where(pos > 0, torch.cat((torch.zeros_like(h[:, :1]), h[:, :-1]), 1), 0.0)
        out["dgate"] = torch.where(pos >= 0, g * (h_prev - x) * f * keep, 0.0).to(s["x"].dtype)
        out["dx"] = torch.where(pos >= 0, g * keep, 0.0).to(s["x"].dtype)
    return out


def _plain_attention(c, s):
    b, t, h, hkv, d = c["b"], c["t"], c["h"], c["hkv"], c["d"]
    dt, scale = s["q"].dtype, 1.0 / math.sqrt(d)

    def heads(x, n):  # [b, t, hkv * n, d] -> [b, hkv, n, t, d]
        return x.float().reshape(b, t, hkv, n, d).permute(0, 2, 3, 1, 4)

    def back(x, n):
        return x.permute(0, 3, 1, 2, 4).reshape(b, t, hkv * n, d).to(dt)

    q, k, v = heads(s["q"], h // hkv), heads(s["k"], 1), heads(s["v"], 1)
    slot = torch.arange(t, device=q.device)
    first = torch.where(s["pos"] >= 0, slot - s["pos"], -1)
    apart = slot[:, None] - slot[None, :]
    seen = (first[:, :, None] == first[:, None, :]) & (first >= 0)[:, :, None]
    if c["causal"]:
        seen = seen & (apart >= 0)
    if c["window"]:
        seen = seen & (apart.abs() < c["window"])
    hidden = ~seen[:, None, None]
    x = (q @ k.transpose(-1, -2)).mul_(scale)
    if c["cap"]:
        th = (x / c["cap"]).tanh_()
        x = th * c["cap"]
    if c["slopes"]:
        x = x - s["slopes"].reshape(1, hkv, h // hkv, 1, 1) * apart.abs().float()
    x = x.masked_fill_(hidden, -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).reshape(b, h, t)
    p = p.div_(torch.where(total > 0, total, 1.0))
    out = p @ v
    res = {"out": back(out, h // hkv), "lse": lse}
    if c["train"]:
        do = heads(s["dout"], h // hkv)
        do = torch.where((first >= 0)[:, None, None, :, None], do, 0.0)
        res["dv"] = back((p.transpose(-1, -2) @ do).sum(2, keepdim=True), 1)
        ds = (do @ v.transpose(-1, -2)).sub_((do * out).sum(-1, keepdim=True)).mul_(p)
        if c["cap"]:
            ds = ds.mul_(th.square_().neg_().add_(1.0))
        res["dq"] = back((ds @ k).mul_(scale), h // hkv)
        res["dk"] = back((ds.transpose(-1, -2) @ q).sum(2, keepdim=True).mul_(scale), 1)
    return res


_own = {"rotary": _own_rotary, "recurrence": _own_recurrence, "attention": _own_attention}
_plain = {"rotary": _plain_rotary, "recurrence": _plain_recurrence, "attention": _plain_attention}


# ---- the work of a pass -------------------------------------------------------------------------------------------

def _pairs(case):
    """Query-key pairs of one head over all blocks, for a fixed draw of the sequence lengths."""
    total = 0
    for here in _blocks(case, 0):
        n = np.asarray(here, dtype=np.int64)
        w = np.minimum(n, case["window"]) if case["window"] else n
        one_side = w * (w + 1) // 2 + (n - w) * w  # j in (i - w, i]
        total += int((one_side if case["causal"] else 2 * one_side - n).sum())
    return total


def work(case):
    b, t, d = case["b"], case["t"], case["d"]
    size = 4 if case["dtype"] == "fp32" else 2
    pos = 4 * b * t
    if case["op"] == "rotary":
        n = b * t * case["h"]
        return {"bytes": 2 * n * d * size + pos + 2 * case["rot"], "flops": 3 * n * case["rot"]}
    if case["op"] == "recurrence":
        n = b * t * d
        return {"bytes": n * size * (6 if case["train"] else 3) + pos, "flops": n * (24 if case["train"] else 9)}
    rows, kv = b * t * case["h"], b * t * case["hkv"]
    moved = (4 if case["train"] else 2) * (rows + kv) * d * size + 4 * rows + pos  # q, k, v, out; dout, dq, dk, dv; lse
    return {"bytes": moved, "flops": (14 if case["train"] else 4) * d * case["h"] * _pairs(case)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotary": _exact_rotary, "recurrence": _exact_recurrence, "attention": _exact_attention}[case["op"]](
        case, s, _blocks(case, seed))


def _exact_rotary(c, s, blocks):
    x, n = s["x"].double(), c["rot"] // 2
    y = x.clone()
    at = (lambda i: (slice(0, 2 * n, 2), slice(1, 2 * n, 2))[i]) if c["interleaved"] else \
        (lambda i: (slice(0, n), slice(n, 2 * n))[i])
    for b, here in enumerate(blocks):
        fill = sum(here)
        where = torch.cat([torch.arange(m) for m in here]).to(x.device).double()
        turn = torch.polar(torch.full((fill, n), c["factor"], dtype=torch.float64, device=x.device),
                           torch.outer(where, s["inv_freq"].double()))
        if c["grad"]:
            turn = turn.conj()
        z = torch.complex(x[b, :fill, :, at(0)], x[b, :fill, :, at(1)]) * turn[:, None]
        y[b, :fill, :, at(0)], y[b, :fill, :, at(1)] = z.real, z.imag
    return {"y": y}


def _exact_recurrence(c, s, blocks):
    pos = s["pos"].cpu()
    gate, x = s["gate"].double(), s["x"].double()
    f = 1.0 / (1.0 + (-gate).exp())
    keep = 1.0 / (1.0 + gate.exp())
    h = torch.zeros_like(x)
    starts, empty = (pos == 0).to(x.device), (pos < 0).to(x.device)
    live, go = (~empty).double()[..., None], (~empty & ~starts).double()[..., None]
    last = torch.zeros_like(x[:, 0])
    push, pull = keep * x * live, f * go
    for i in range(c["t"]):
        last = torch.addcmul(push[:, i], pull[:, i], last)
        h[:, i] = last
    out = {"h": h}
    if c["train"]:
        dh = s["dh"].double() * live
        g, carry = torch.zeros_like(x), torch.zeros_like(last)
        for i in range(c["t"] - 1, -1, -1):
            carry = dh[:, i] + carry
            g[:, i] = carry
            carry = carry * pull[:, i]
        before = torch.zeros_like(h)
        before[:, 1:] = h[:, :-1]
        before *= go
        out["dgate"] = g * (before - x) * f * keep * live
        out["dx"] = g * keep * live
    return out


def _exact_attention(c, s, blocks):
    if sum(n * n for here in blocks for n in here) * c["h"] > 1.3e9:
        return None
    h, hkv, d = c["h"], c["hkv"], c["d"]
    res = {n: torch.zeros(s[n].shape, dtype=torch.float64, device=s["q"].device)
           for n in (("out", "dq", "dk", "dv") if c["train"] else ("out",))}
    res["lse"] = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, here in enumerate(blocks):
        at = 0
        for n in here:
            rows = slice(at, at + n)
            at += n
            i = torch.arange(n, device=s["q"].device)
            off = (i[:, None] - i[None, :]).double()
            bad = torch.zeros_like(off, dtype=torch.bool)
            if c["causal"]:
                bad |= off < 0
            if c["window"]:
                bad |= off.abs() >= c["window"]
            for kv in range(hkv):
                k = s["k"][b, rows, kv].double().requires_grad_(c["train"])
                v = s["v"][b, rows, kv].double().requires_grad_(c["train"])
                own_heads = range(kv * (h // hkv), (kv + 1) * (h // hkv))
                q = s["q"][b, rows, own_heads.start:own_heads.stop].double().transpose(0, 1).contiguous()
                q.requires_grad_(c["train"])
                score = torch.einsum("hid,jd->hij", q, k) / math.sqrt(d)
                if c["cap"]:
                    score = torch.tanh(score / c["cap"]) * c["cap"]
                if c["slopes"]:
                    score = score - s["slopes"][own_heads.start:own_heads.stop].double()[:, None, None] * off.abs()
                score = score.masked_fill(bad, -math.inf)
                res["lse"][b, own_heads.start:own_heads.stop, rows] = torch.logsumexp(score.detach(), -1)
                o = torch.softmax(score, -1) @ v
                res["out"][b, rows, own_heads.start:own_heads.stop] = o.detach().transpose(0, 1)
                if c["train"]:
                    do = s["dout"][b, rows, own_heads.start:own_heads.stop].double().transpose(0, 1)
                    dq, dk, dv = torch.autograd.grad(o, (q, k, v), do)
                    res["dq"][b, rows, own_heads.start:own_heads.stop] = dq.transpose(0, 1)
                    res["dk"][b, rows, kv], res["dv"][b, rows, kv] = dk, dv
    return res
