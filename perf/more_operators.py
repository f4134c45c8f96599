"""Cases for the operators of a state-space model over packed batches, and for rotary positions with several axes: layer norm,
a short causal convolution, a selective state-space scan (the last two for training, for prompts and for single tokens).

A packed batch holds several sequences in each block of `t` slots; `pos[b, s]` is a slot's position in its sequence and
-1 on padding, as bload_pack writes it.  Padding slots give 0 everywhere (rotary: their input) and have no influence.

  norm         y = (x - mean) / sqrt(var + eps) * weight + bias over the channels of a frame; gradients of x, weight, bias.
  conv         u_s = bias + sum_j weight[:, taps - 1 - j] x_{s - j} over the j < taps that stay in the sequence; y = u or
               u * sigmoid(u); gradients of x, weight, bias.
  conv_step    the same for one new token of each of n sequences, whose last taps - 1 inputs are kept in a state.
  scan         delta = softplus(dt + dt_bias); per channel and state n, h_s = exp(delta a_n) h_{s-1} + delta b_n x with
               h = 0 in front of a sequence; y = (sum_n c_n h_n + d x) * (z sigmoid(z) if given); all gradients.
  scan_step    the same for one new token of each of n sequences, whose h is kept in a state.
  rotary_axes  every pair of a head turned by coordinate[axis of the pair] * inv_freq[pair].

`own` selects between the framework's calls and plain torch operations in 32 bits (64 for angles).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
AXES = 3


def listed():
    return [
        # Toy clips (blocks of 64 slots): one batch is a few hundred kilobytes, so this is the latency of a call.
        {"name": "norm toy", "op": "norm", "train": False, "b": 8, "t": 64, "c": 512, "dtype": "fp16", "docs": "toy"},
        # Training step on token blocks, 2048 channels: memory.
        {"name": "norm train tokens", "op": "norm", "train": True, "b": 16, "t": 4096, "c": 2048, "dtype": "bf16",
         "docs": "tokens"},
        # Residual stream in 32 bits with an odd number of channels, video features in heavy-tailed lengths.
        {"name": "norm train odd", "op": "norm", "train": True, "b": 4, "t": 5003, "c": 1027, "dtype": "fp32",
         "docs": "heavy"},
        # The convolution in front of the scan in a training step on token blocks.
        {"name": "conv train tokens", "op": "conv", "train": True, "b": 8, "t": 4096, "c": 2048, "taps": 4, "silu": True,
         "dtype": "bf16", "docs": "tokens"},
        # One token of each of 256 sequences: the convolution's part of a decoding step.
        {"name": "conv step", "op": "conv_step", "n": 256, "c": 4096, "taps": 4, "silu": True, "dtype": "fp16"},
        # One batch of toy clips through a small layer: latency.
        {"name": "scan toy", "op": "scan", "train": False, "b": 8, "t": 64, "c": 256, "n": 16, "z": True, "last": False,
         "dtype": "fp16", "docs": "toy"},
        # Prompts packed into token blocks, whose last states start the generation of single tokens.
        {"name": "scan prompts", "op": "scan", "train": False, "b": 8, "t": 4096, "c": 2048, "n": 16, "z": True, "last": True,
         "dtype": "bf16", "docs": "tokens"},
        # Training step of the heavy-tailed workload: 4 blocks of 10,000 frames.
        {"name": "scan train heavy", "op": "scan", "train": True, "b": 4, "t": 10000, "c": 1024, "n": 16, "z": True,
         "last": False, "dtype": "bf16", "docs": "heavy"},
        # One long sequence, few and odd channels, 32 bits: the time axis is all there is to split.
        {"name": "scan train long", "op": "scan", "train": True, "b": 1, "t": 20011, "c": 509, "n": 8, "z": False,
         "last": False, "dtype": "fp32", "docs": "single"},
        # One token of each of 256 sequences: the scan's part of a decoding step.
        {"name": "scan step", "op": "scan_step", "n": 256, "c": 4096, "states": 16, "z": True, "dtype": "bf16"},
        # Queries and keys of video tokens (time, height, width), sections of a head of 128 for the three axes.
        {"name": "rotary axes video", "op": "rotary_axes", "grad": False, "b": 16, "t": 4096, "h": 20, "d": 128, "rot": 128,
         "interleaved": False, "sections": True, "dtype": "bf16", "docs": "tokens"},
        # Gradient on part of a head in 32 bits, neighbours as pairs, the axes taking turns along the pairs.
        {"name": "rotary axes grad", "op": "rotary_axes", "grad": True, "b": 4, "t": 5003, "h": 9, "d": 80, "rot": 60,
         "interleaved": True, "sections": False, "dtype": "fp32", "docs": "heavy"},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "conv", "conv", "conv_step", "scan", "scan", "scan", "scan_step", "rotary_axes", "rotary_axes"])
    dtype = rng.choice(["fp32", "fp16", "bf16"])
    wide = 2 if dtype == "fp32" else 1
    case = {"op": op, "dtype": dtype}
    if op in ("conv_step", "scan_step"):
        c = _log_int(rng, 1, 8192)
        if rng.random() < 0.7:
            c = -(-c // 8) * 8
        n = _log_int(rng, 1, max(1, min(1024, 256 * 4096 // c // wide)))
        if op == "conv_step":
            return dict(case, n=n, c=c, taps=rng.choice([2, 3, 4, 4, 6, 8]), silu=rng.random() < 0.7)
        states = rng.choice([16, 16, 8, rng.randint(1, 64)])
        return dict(case, n=max(1, n * 16 // max(16, states)), c=c, states=states, z=rng.random() < 0.5)
    case["docs"] = rng.choice(["toy", "features", "tokens", "heavy", "single"])
    t = _log_int(rng, 1, 16384)
    if op == "rotary_axes":
        d = 8 * rng.randint(1, 16) if rng.random() < 0.7 else rng.randint(2, 128)
        rows = _log_int(rng, 1, max(1, 16 * 4096 * 20 * 128 // (t * d * wide)))  # blocks x heads
        h = min(rows, rng.randint(1, 32))
        return dict(case, grad=rng.random() < 0.5, b=max(1, rows // h), t=t, h=h, d=d,
                    rot=min(d // 2 * 2, 2 * rng.randint(1, max(1, d // 2))), interleaved=rng.random() < 0.5,
                    sections=rng.random() < 0.5)
    c = _log_int(rng, 16, 8192) if op == "norm" else _log_int(rng, 1, 4096)  # (of 2 channels the gradient is all cancellation)
    if rng.random() < 0.7:
        c = -(-c // 8) * 8
    train = rng.random() < 0.6
    if op == "scan":
        n = rng.choice([16, 16, 8, rng.randint(1, 64)])
        room = (4 * 10000 * 1024 * 16 if train else 8 * 4096 * 2048 * 16) // wide
        t = min(t, max(1, room // (c * n)))
        b = _log_int(rng, 1, max(1, min(64, room // (t * c * n))))
        return dict(case, train=train, b=b, t=t, c=c, n=n, z=rng.random() < 0.5, last=not train and rng.random() < 0.5)
    room = (16 if op == "norm" else 8) * 4096 * 2048 // wide
    b = _log_int(rng, 1, max(1, min(256, room // (t * c))))
    case.update(train=train, b=b, t=t, c=c)
    return case if op == "norm" else dict(case, taps=rng.choice([2, 3, 4, 4, 6, 8]), silu=rng.random() < 0.7)


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
    rng = np.random.default_rng(0 if case.get("last") else seed)  # (a state per sequence: as many whatever the seed)
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


def _tables(case, blocks):
    """(positions, sequence numbers) of the slots, -1 on padding."""
    pos = np.full((case["b"], case["t"]), -1, np.int32)
    seq = np.full((case["b"], case["t"]), -1, np.int32)
    k = 0
    for row, ids, here in zip(pos, seq, blocks):
        s = 0
        for n in here:
            row[s:s + n] = np.arange(n, dtype=np.int32)
            ids[s:s + n] = k
            k += 1
            s += n
    return pos, seq


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dt, f32 = TYPES[case["dtype"]], torch.float32
    op = case["op"]
    state = {"case": dict(case)}
    step = op in ("conv_step", "scan_step")

    def normal(*shape, mean=0.0, std=1.0, dtype=dt):
        return torch.empty(shape, dtype=f32, device=dev).normal_(mean, std, generator=g).to(dtype)

    def uniform(*shape, lo, hi):
        return torch.empty(shape, dtype=f32, device=dev).uniform_(lo, hi, generator=g)

    def empty(x, dtype=None):
        return torch.empty(x.shape, dtype=dtype or x.dtype, device=dev)

    if step:
        rows = (case["n"],)
        # requests at any point of their sequence; some have just begun, a few places of the batch are free
        at = np.random.default_rng(seed).choice(np.array([-1, 0, 1, 2, 700], np.int32), case["n"], p=[0.05, 0.1, 0.1, 0.1, 0.65])
        state["pos"] = torch.from_numpy(at).to(dev)
    else:
        rows = (case["b"], case["t"])
        blocks = _blocks(case, seed)
        pos, seq = _tables(case, blocks)
        state["pos"] = torch.from_numpy(pos).to(dev)
    if op == "rotary_axes":
        n = case["rot"] // 2
        # axis of every pair: sections of a quarter for the time and the rest for height and width, or in turn
        i = torch.arange(n)
        state["axis"] = (torch.where(i < n // 4, 0, torch.where(i < n // 4 + (n - n // 4) // 2, 1, 2)) if case["sections"]
                         else i % AXES).to(torch.int32).to(dev)
        state["inv_freq"] = (10000.0 ** (-i.double() / max(n, 1))).float().to(dev)
        # frames of 18 x 32 patches, behind some earlier part of the stream: far coordinates along the time
        p = state["pos"].clamp(min=0)
        state["coords"] = torch.stack((p // 576 + 20000, p % 576 // 32, p % 32)).to(torch.int32).contiguous()
        state["x"] = normal(*rows, case["h"], case["d"])
        state["y"] = empty(state["x"])
        return state
    c = case["c"]
    state["x"] = normal(*rows, c)
    state["y"] = empty(state["x"])
    train = case.get("train", False)
    if train:
        state["dy"], state["dx"] = normal(*rows, c), empty(state["x"])
    if op == "norm":
        state["x"] = (state["x"].float() * 2.0 + 0.5).to(dt)
        state["weight"], state["bias"] = normal(c, mean=1.0, std=0.1, dtype=f32), normal(c, std=0.1, dtype=f32)
        state["dweight"], state["dbias"] = empty(state["weight"]), empty(state["bias"])
    elif op in ("conv", "conv_step"):
        k = case["taps"]
        state["weight"], state["bias"] = normal(c, k, std=k ** -0.5, dtype=f32), normal(c, std=0.1, dtype=f32)
        if step:
            state["state"] = normal(case["n"], k - 1, c)
            state["next"] = empty(state["state"])
        else:
            state["dweight"], state["dbias"] = empty(state["weight"]), empty(state["bias"])
    else:
        n = case["states"] if step else case["n"]
        state["dt"] = normal(*rows, c, std=0.7)
        state["b"], state["c"] = normal(*rows, n), normal(*rows, n)
        state["a"] = -torch.arange(1, n + 1, device=dev, dtype=f32) * normal(c, n, std=0.1, dtype=f32).exp()
        delta = uniform(c, lo=math.log(0.001), hi=math.log(0.1)).exp()
        state["dt_bias"] = delta + torch.log(-torch.expm1(-delta))  # softplus(dt_bias) = delta
        state["d"] = normal(c, mean=1.0, std=0.2, dtype=f32)
        state["z"] = normal(*rows, c) if case["z"] else None
        if step:
            state["state"] = normal(case["n"], c, n, std=0.3, dtype=f32)
            state["next"] = empty(state["state"])
        elif case["last"]:
            state["seq_id"] = torch.from_numpy(seq).to(dev)
            state["last"] = torch.zeros((sum(map(len, blocks)), c, n), dtype=f32, device=dev)
        if train:
            for name in ("dt", "b", "c", "a", "dt_bias", "d"):
                state["d" + name] = empty(state[name])
            state["dz"] = empty(state["z"]) if case["z"] else None
    return state


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["op"]](case, state)


def _own_norm(c, s):
    import paper_2310_10879_b200 as B
    if not c["train"]:
        B.bload_norm(s["pos"], s["x"], s["y"], s["weight"], s["bias"], eps=EPS)
        return {"y": s["y"]}
    stats, work = B.bload_norm_buffers(s["pos"], s["x"])  # means and deviations kept for the backward pass, and scratch
    B.bload_norm(s["pos"], s["x"], s["y"], s["weight"], s["bias"], stats, eps=EPS)
    B.bload_norm_grad(s["pos"], s["x"], stats, s["dy"], s["dx"], s["weight"], s["dweight"], s["dbias"], work)
    return {n: s[n] for n in ("y", "dx", "dweight", "dbias")}


def _own_conv(c, s):
    import paper_2310_10879_b200 as B
    B.bload_conv(s["pos"], s["x"], s["y"], s["weight"], s["bias"], silu=c["silu"])
    if not c["train"]:
        return {"y": s["y"]}
    work = B.bload_conv_buffers(s["pos"], s["x"], s["weight"])
    B.bload_conv_grad(s["pos"], s["x"], s["dy"], s["dx"], s["weight"], s["dweight"], s["bias"], s["dbias"], silu=c["silu"],
                      work=work)
    return {n: s[n] for n in ("y", "dx", "dweight", "dbias")}


def _own_conv_step(c, s):
    import paper_2310_10879_b200 as B
    B.bload_conv_step(s["pos"], s["state"], s["x"], s["y"], s["weight"], s["bias"], silu=c["silu"], next_state=s["next"])
    return {"y": s["y"], "next": s["next"]}


def _own_scan(c, s):
    import paper_2310_10879_b200 as B
    carry, work = B.bload_scan_buffers(s["pos"], s["x"], s["a"], gradient=c["train"])  # states kept for the backward pass
    more = {"d": s["d"], "dt_bias": s["dt_bias"], "z": s["z"], "work": work}
    kept = {"seq_id": s["seq_id"], "last": s["last"]} if c["last"] else {}
    B.bload_scan(s["pos"], s["x"], s["dt"], s["a"], s["b"], s["c"], s["y"], carry=carry, **kept, **more)
    if not c["train"]:
        return {"y": s["y"], "last": s["last"]} if c["last"] else {"y": s["y"]}
    B.bload_scan_grad(s["pos"], s["x"], s["dt"], s["a"], s["b"], s["c"], carry, s["dy"], s["dx"], s["ddt"], s["da"], s["db"],
                      s["dc"], dd=s["dd"], ddt_bias=s["ddt_bias"], dz=s["dz"], **more)
    return {n: s[n] for n in ("y", "dx", "ddt", "da", "db", "dc", "dd", "ddt_bias", "dz") if s[n] is not None}


def _own_scan_step(c, s):
    import paper_2310_10879_b200 as B
    B.bload_scan_step(s["pos"], s["state"], s["x"], s["dt"], s["a"], s["b"], s["c"], s["y"], d=s["d"], dt_bias=s["dt_bias"],
                      z=s["z"], next_state=s["next"])
    return {"y": s["y"], "next": s["next"]}


def _own_rotary_axes(c, s):
    import paper_2310_10879_b200 as B
    call = B.bload_rotary_axes_grad if c["grad"] else B.bload_rotary_axes
    call(s["pos"], s["coords"], s["axis"], s["x"], s["y"], s["inv_freq"], interleaved=c["interleaved"])
    return {"y": s["y"]}


def _plain_norm(c, s):
    dt, live = s["x"].dtype, (s["pos"] >= 0)[..., None]
    x = torch.where(live, s["x"].float(), 0.0)
    x = x - x.mean(-1, keepdim=True)
    rstd = 1.0 / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    xhat = x * rstd
    out = {"y": torch.where(live, xhat * s["weight"] + s["bias"], 0.0).to(dt)}
    if c["train"]:
        dy = torch.where(live, s["dy"].float(), 0.0)
        g = dy * s["weight"]
        dx = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
        out["dx"] = torch.where(live, dx, 0.0).to(dt)
        out["dweight"], out["dbias"] = (dy * xhat).sum((0, 1)), dy.sum((0, 1))
    return out


def _back(x, j):
    """x[:, s - j], zeros in front."""
    return torch.cat((torch.zeros_like(x[:, :j]), x[:, :x.shape[1] - j]), 1) if j else x


def _ahead(x, j):
    """x[:, s + j], zeros behind."""
    return torch.cat((x[:, j:], torch.zeros_like(x[:, :j])), 1) if j else x


def _plain_conv(c, s):
    dt, k = s["x"].dtype, c["taps"]
    pos = s["pos"][..., None]
    live, w = pos >= 0, s["weight"]
    x = torch.where(live, s["x"].float(), 0.0)
    taps = [torch.where(pos >= j, _back(x, j), 0.0) for j in range(min(k, c["t"]))]  # tap j: the input j slots back
    u = s["bias"] + sum(w[:, k - 1 - j] * v for j, v in enumerate(taps))
    gate = torch.sigmoid(u) if c["silu"] else torch.ones_like(u)
    out = {"y": torch.where(live, u * gate, 0.0).to(dt)}
    if c["train"]:
        du = torch.where(live, s["dy"].float(), 0.0)
        if c["silu"]:
            du = du * gate * (1.0 + u * (1.0 - gate))
        out["dx"] = sum(w[:, k - 1 - j] * _ahead(torch.where(pos >= j, du, 0.0), j) for j in range(len(taps))).to(dt)
        zero = torch.zeros_like(w[:, 0])
        out["dweight"] = torch.stack([(du * taps[k - 1 - i]).sum((0, 1)) if k - 1 - i < len(taps) else zero
                                      for i in range(k)], 1)
        out["dbias"] = du.sum((0, 1))
    return out


def _plain_conv_step(c, s):
    dt, pos = s["x"].dtype, s["pos"][:, None]
    k = c["taps"]
    window = torch.cat((s["state"].float(), s["x"].float()[:, None]), 1)  # [n, taps, c], oldest first
    back = torch.arange(k - 1, -1, -1, device=pos.device)
    window = torch.where((pos >= back)[..., None], window, 0.0)  # inputs in front of the sequence
    u = s["bias"] + (window * s["weight"].t()).sum(1)
    if c["silu"]:
        u = u * torch.sigmoid(u)
    return {"y": torch.where(pos >= 0, u, 0.0).to(dt), "next": torch.where((pos >= 0)[..., None], window[:, 1:], s["state"].float()).to(dt)}


def _linear_scan(a, u):
    """h[s] = a[s] * h[s - 1] + u[s] along dim 1, by doubling the reach of every slot."""
    k = 1
    while k < a.shape[1]:
        u = torch.cat((u[:, :k], u[:, k:] + a[:, k:] * u[:, :-k]), 1)
        a = torch.cat((a[:, :k], a[:, k:] * a[:, :-k]), 1)
        k *= 2
    return u


def _softplus(v):
    return torch.where(v > 20.0, v, torch.log1p(torch.exp(v.clamp(max=20.0))))


def _plain_scan(c, s):
    dt, pos = s["x"].dtype, s["pos"][..., None]
    live, A = pos >= 0, s["a"]

    def read(name):
        return torch.where(live, s[name].float(), 0.0)

    x, B, C = read("x"), read("b")[:, :, None], read("c")[:, :, None]
    raw = s["dt"].float() + s["dt_bias"]
    delta = torch.where(live, _softplus(raw), 0.0)
    a = torch.where((pos > 0)[..., None], torch.exp(delta[..., None] * A), 0.0)
    h = _linear_scan(a, (delta * x)[..., None] * B)
    y = (h * C).sum(-1) + s["d"] * x
    z = read("z") if c["z"] else None
    gate = torch.sigmoid(z) if c["z"] else None
    out = {"y": (y * z * gate if c["z"] else y).to(dt)}
    if c["last"]:
        seq = s["seq_id"]
        follows = torch.cat((seq[:, 1:], torch.full_like(seq[:, :1], -1)), 1)
        ends = (seq >= 0) & (follows != seq)
        last = torch.zeros_like(s["last"])
        last[seq[ends].long()] = h[ends]
        out["last"] = last
    if not c["train"]:
        return out
    dy = read("dy")
    do = dy * z * gate if c["z"] else dy
    if c["z"]:
        out["dz"] = (dy * y * gate * (1.0 + z * (1.0 - gate))).to(dt)
    a_next = torch.cat((a[:, 1:], torch.zeros_like(a[:, :1])), 1)
    out["dc"] = (h * do[..., None]).sum(2).to(dt)
    g = _linear_scan(a_next.flip(1), (do[..., None] * C).flip(1)).flip(1)
    del a_next
    out["db"] = (g * (delta * x)[..., None]).sum(2).to(dt)
    through = g * a * torch.cat((torch.zeros_like(h[:, :1]), h[:, :-1]), 1)  # (a is 0 where a sequence starts)
    out["da"] = (through * delta[..., None]).sum((0, 1))
    gb = (g * B).sum(-1)
    ddt = (x * gb + (through * A).sum(-1)) * torch.sigmoid(raw)
    ddt = torch.where(live, ddt, 0.0)
    out["ddt"], out["ddt_bias"] = ddt.to(dt), ddt.sum((0, 1))
    out["dx"], out["dd"] = (delta * gb + s["d"] * do).to(dt), (do * x).sum((0, 1))
    return out


def _plain_scan_step(c, s):
    dt, pos = s["x"].dtype, s["pos"][:, None]
    x, z = s["x"].float(), s["z"]
    delta = _softplus(s["dt"].float() + s["dt_bias"])
    h = torch.where((pos > 0)[..., None], s["state"], 0.0) * torch.exp(delta[..., None] * s["a"])
    h = h + (delta * x)[..., None] * s["b"].float()[:, None]
    y = (h * s["c"].float()[:, None]).sum(-1) + s["d"] * x
    if c["z"]:
        y = y * z.float() * torch.sigmoid(z.float())
    return {"y": torch.where(pos >= 0, y, 0.0).to(dt), "next": torch.where((pos >= 0)[..., None], h, s["state"])}


def _plain_rotary_axes(c, s):
    x, n = s["x"].float(), c["rot"] // 2
    at = s["coords"].permute(1, 2, 0)[..., s["axis"].long()]  # the coordinate of every pair
    angle = at.double() * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    if c["grad"]:
        sin = -sin
    if c["interleaved"]:
        u, w = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
        y = torch.stack((u * cos - w * sin, w * cos + u * sin), -1).flatten(-2)
    else:
        u, w = x[..., :n], x[..., n:2 * n]
        y = torch.cat((u * cos - w * sin, w * cos + u * sin), -1)
    y = torch.cat((y, x[..., 2 * n:]), -1)
    return {"y": torch.where((s["pos"] >= 0)[..., None, None], y, x).to(s["x"].dtype)}


_own = {"norm": _own_norm, "conv": _own_conv, "conv_step": _own_conv_step, "scan": _own_scan, "scan_step": _own_scan_step,
        "rotary_axes": _own_rotary_axes}
_plain = {"norm": _plain_norm, "conv": _plain_conv, "conv_step": _plain_conv_step, "scan": _plain_scan,
          "scan_step": _plain_scan_step, "rotary_axes": _plain_rotary_axes}


# ---- the work of a pass -------------------------------------------------------------------------------------------

def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    op = case["op"]
    if op == "conv_step":
        n, k = case["n"] * case["c"], case["taps"]
        return {"bytes": n * size * (2 + 2 * (k - 1)) + 4 * case["c"] * (k + 1) + 4 * case["n"], "flops": n * (2 * k + 6)}
    if op == "scan_step":
        n, m = case["n"] * case["c"], case["states"]
        moved = n * (8 * m + size * (4 if case["z"] else 3)) + 2 * case["n"] * m * size + 4 * case["c"] * (m + 2) + 4 * case["n"]
        return {"bytes": moved, "flops": n * (8 * m + 20)}
    slots = case["b"] * case["t"]
    if op == "rotary_axes":
        n = slots * case["h"]
        return {"bytes": 2 * n * case["d"] * size + 4 * slots * (1 + AXES) + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    n, train = slots * case["c"], case["train"]
    if op == "norm":  # x, y; dy, dx
        return {"bytes": n * size * (4 if train else 2) + 4 * slots + 4 * case["c"] * (4 if train else 2), "flops": n * (20 if train else 8)}
    if op == "conv":
        k = case["taps"]
        return {"bytes": n * size * (4 if train else 2) + 4 * slots + 4 * case["c"] * (k + 1) * (2 if train else 1),
                "flops": n * ((8 * k + 16) if train else (2 * k + 6))}
    m = case["n"]
    tensors = (6 if train else 3) + ((2 if train else 1) if case["z"] else 0)  # x, dt, y; dy, dx, ddt; z, dz
    moved = n * size * tensors + slots * m * size * (4 if train else 2) + 4 * slots + 4 * case["c"] * (m + 2) * (2 if train else 1)
    if case["last"]:
        moved += 4 * slots + 4 * case["c"] * m * sum(map(len, _blocks(case, 0)))  # sequence numbers, last states
    return {"bytes": moved, "flops": n * m * (26 if train else 8)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "scan" and case["b"] * case["t"] * case["c"] * case["n"] > 1.2e9:
        return None
    s = prepare(case, seed)
    wide = {n: v.double() if torch.is_tensor(v) and v.is_floating_point() else v for n, v in s.items()
            if n not in ("y", "dx", "next", "last")}
    return {"norm": _exact_norm, "conv": _exact_conv, "conv_step": _exact_conv_step, "scan": _exact_scan,
            "scan_step": _exact_scan_step, "rotary_axes": _exact_rotary_axes}[case["op"]](case, wide, s)


def _exact_norm(c, w, s):
    rows = (s["pos"] >= 0).reshape(-1).nonzero()[:, 0]  # the frames, without the padding
    x = w["x"].reshape(-1, c["c"])[rows]
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    unit = (x - mean) / torch.sqrt(var + EPS)

    def spread(v):
        return torch.zeros((c["b"] * c["t"], c["c"]), dtype=torch.float64, device=v.device).index_copy_(0, rows, v).reshape(s["x"].shape)

    out = {"y": spread(torch.addcmul(w["bias"], unit, w["weight"]))}
    if c["train"]:
        dy = w["dy"].reshape(-1, c["c"])[rows]
        g = dy * w["weight"]
        along = (g * unit).sum(-1, keepdim=True) / c["c"]
        out["dx"] = spread((g - g.sum(-1, keepdim=True) / c["c"] - unit * along) / torch.sqrt(var + EPS))
        out["dweight"], out["dbias"] = torch.einsum("rc,rc->c", dy, unit), torch.einsum("rc->c", dy)
    return out


def _exact_conv(c, w, s):
    """Every sequence padded in front and behind by itself; sequences of a batch side by side in one long row with gaps."""
    k = c["taps"]
    pos = s["pos"].reshape(-1).cpu().numpy()
    frames = np.flatnonzero(pos >= 0)
    starts = np.cumsum(pos[frames] == 0)  # 1, 2, ... per sequence
    where = torch.from_numpy(np.arange(frames.size) + (k - 1) * starts).to(s["x"].device)
    frames = torch.from_numpy(frames).to(s["x"].device)
    total = int(frames.numel() + (k - 1) * (int(starts[-1]) if starts.size else 0) + (k - 1))
    row = torch.zeros((total, c["c"]), dtype=torch.float64, device=s["x"].device)
    row[where] = w["x"].reshape(-1, c["c"])[frames]
    u = w["bias"].expand(frames.numel(), c["c"]).clone()
    for i in range(k):
        u += w["weight"][:, i] * row[where - (k - 1) + i]
    sig = 1.0 / (1.0 + torch.exp(-u))

    def spread(v):
        return torch.zeros((c["b"] * c["t"], c["c"]), dtype=torch.float64, device=v.device).index_copy_(0, frames, v).reshape(s["x"].shape)

    out = {"y": spread(u * sig if c["silu"] else u)}
    if c["train"]:
        du = w["dy"].reshape(-1, c["c"])[frames]
        if c["silu"]:
            du = du * (sig + u * sig * (1.0 - sig))
        out["dweight"] = torch.stack([(du * row[where - (k - 1) + i]).sum(0) for i in range(k)], 1)
        out["dbias"] = du.sum(0)
        drow = torch.zeros_like(row)
        for i in range(k):
            drow.index_add_(0, where - (k - 1) + i, du * w["weight"][:, i])
        out["dx"] = spread(drow[where])
    return out


def _exact_conv_step(c, w, s):
    k, y, kept = c["taps"], torch.zeros_like(w["x"]), w["state"].clone()
    for p in sorted(set(s["pos"].tolist()) - {-1}):
        rows = (s["pos"] == p).nonzero()[:, 0]
        have = min(p, k - 1)  # inputs in front of this one that are the sequence's own
        seen = torch.cat((torch.zeros((rows.numel(), k - 1 - have, c["c"]), dtype=torch.float64, device=rows.device),
                          w["state"][rows][:, k - 1 - have:], w["x"][rows][:, None]), 1)
        u = torch.einsum("nkc,ck->nc", seen, w["weight"]) + w["bias"]
        y[rows] = u / (1.0 + torch.exp(-u)) if c["silu"] else u
        kept[rows] = seen[:, 1:]
    return {"y": y, "next": kept}


def _exact_scan(c, w, s):
    pos = s["pos"]
    dev, f64 = pos.device, torch.float64
    b, t, ch, n = c["b"], c["t"], c["c"], c["n"]
    x, A = w["x"], w["a"]
    raw = w["dt"] + w["dt_bias"]
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    h = torch.zeros((b, ch, n), dtype=f64, device=dev)
    kept = torch.zeros((t, b, ch, n), dtype=f64, device=dev) if c["train"] else None
    y = torch.zeros_like(x)
    cols = pos.t().contiguous()
    here, goes = (cols >= 0).double()[:, :, None, None], (cols > 0).double()[:, :, None, None]
    last = torch.zeros(s["last"].shape, dtype=f64, device=dev) if c["last"] else None
    ends = [[] for _ in range(t)]
    if c["last"]:
        seq = s["seq_id"].cpu().numpy()
        for q in range(b):
            for i in range(t):
                if seq[q, i] >= 0 and (i + 1 == t or seq[q, i + 1] != seq[q, i]):
                    ends[i].append((q, int(seq[q, i])))
    for i in range(t):
        h = goes[i] * h * torch.exp(delta[:, i, :, None] * A) + here[i] * (delta[:, i] * x[:, i])[:, :, None] * w["b"][:, i, None]
        y[:, i] = torch.matmul(h, w["c"][:, i, :, None])[..., 0]
        if kept is not None:
            kept[i] = h
        for q, k in ends[i]:
            last[k] = h[q]
    live = (pos >= 0)[..., None].double()
    y = (y + w["d"] * x) * live
    sig = 1.0 / (1.0 + torch.exp(-w["z"])) if c["z"] else None
    out = {"y": y * w["z"] * sig if c["z"] else y}
    if c["last"]:
        out["last"] = last
    if not c["train"]:
        return out
    do = w["dy"] * live
    if c["z"]:
        out["dz"] = do * y * (sig + w["z"] * sig * (1.0 - sig))
        do = do * w["z"] * sig
    out["dd"] = (do * x).sum((0, 1))
    dx, ddelta = do * w["d"], torch.zeros_like(x)
    db, dc, dA = torch.zeros_like(w["b"]), torch.zeros_like(w["c"]), torch.zeros((b, ch, n), dtype=f64, device=dev)
    g = torch.zeros((b, ch, n), dtype=f64, device=dev)
    for i in range(t - 1, -1, -1):
        dc[:, i] = torch.matmul(do[:, i, None], kept[i])[:, 0]
        g = g + do[:, i, :, None] * w["c"][:, i, None]
        db[:, i] = torch.matmul((delta[:, i] * x[:, i])[:, None], g)[:, 0]
        gb = torch.matmul(g, w["b"][:, i, :, None])[..., 0]
        dx[:, i] += delta[:, i] * gb
        g = g * torch.exp(delta[:, i, :, None] * A) * goes[i]
        if i:
            flow = g * kept[i - 1]
            dA += flow * delta[:, i, :, None]
            ddelta[:, i] = (flow * A).sum(-1)
        ddelta[:, i] += x[:, i] * gb
    ddt = ddelta * live / (1.0 + torch.exp(-raw))
    out.update(dx=dx * live, ddt=ddt, ddt_bias=ddt.sum((0, 1)), da=dA.sum(0), db=db * live, dc=dc * live)
    return out


def _exact_scan_step(c, w, s):
    keep = (s["pos"] > 0).double()[:, None, None]
    raw = w["dt"] + w["dt_bias"]
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    h = keep * w["state"] * torch.exp(torch.einsum("nc,ck->nck", delta, w["a"])) + torch.einsum("nc,nk->nck", delta * w["x"], w["b"])
    y = torch.einsum("nck,nk->nc", h, w["c"]) + w["d"] * w["x"]
    if c["z"]:
        y = y * w["z"] / (1.0 + torch.exp(-w["z"]))
    free = (s["pos"] < 0).nonzero()[:, 0]
    y[free], h[free] = 0.0, w["state"][free]
    return {"y": y, "next": h}


def _exact_rotary_axes(c, w, s):
    x, n = w["x"], c["rot"] // 2
    y = x.clone()
    first, second = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["interleaved"] else (slice(0, n), slice(n, 2 * n))
    for i, (axis, freq) in enumerate(zip(s["axis"].tolist(), w["inv_freq"].tolist())):
        turn = torch.polar(torch.ones(s["pos"].shape, dtype=torch.float64, device=x.device), s["coords"][axis].double() * freq)
        turn = torch.where(s["pos"] >= 0, turn.conj() if c["grad"] else turn, 1.0)[..., None]
        k, m = range(x.shape[-1])[first][i], range(x.shape[-1])[second][i]
        z = torch.complex(x[..., k], x[..., m]) * turn
        y[..., k], y[..., m] = z.real, z.imag
    return {"y": y}
