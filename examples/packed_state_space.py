"""A small state-space model trained on packed blocks, and single tokens generated from packed prompts.

    python examples/packed_state_space.py [--steps N] [--video]

Every layer is a norm, a projection, a short causal convolution and a selective scan, which read the per-slot positions that
bload_pack writes and stay inside sequences.  --video puts an attention layer in front whose rotary positions have two axes: the
sequences are clips of frames of four patches.  Without it, prompts that were packed into blocks are continued one token at a
time from the states that the convolution and the scan leave behind each of them.
"""
from __future__ import annotations

import argparse
import importlib.util
import os
import sys

import torch
from torch.autograd.function import once_differentiable

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.dirname(HERE))
import paper_2310_10879_b200 as B  # noqa: E402

_spec = importlib.util.spec_from_file_location("packed_layers", os.path.join(HERE, "packed_layers.py"))
layers = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(layers)


def _new(like, shape=None, dtype=None):
    return torch.empty(like.shape if shape is None else shape, dtype=dtype or like.dtype, device=like.device)


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, weight, bias):
        stats, _ = B.bload_norm_buffers(pos, x)
        y = _new(x)
        B.bload_norm(pos, x, y, weight, bias, stats)
        ctx.save_for_backward(x, pos, weight, stats)
        return y

    @staticmethod
    @once_differentiable  # (the gradient calls have no gradients of their own)
    def backward(ctx, dy):
        x, pos, weight, stats = ctx.saved_tensors
        dx, dweight, dbias = _new(x), _new(weight), _new(weight)
        B.bload_norm_grad(pos, x, stats, dy.contiguous(), dx, weight, dweight, dbias, B.bload_norm_buffers(pos, x)[1])
        return dx, None, dweight, dbias


class Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, weight, bias):
        y = _new(x)
        B.bload_conv(pos, x, y, weight, bias)
        ctx.save_for_backward(x, pos, weight, bias)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, pos, weight, bias = ctx.saved_tensors
        dx, dweight, dbias = _new(x), _new(weight), _new(bias)
        B.bload_conv_grad(pos, x, dy.contiguous(), dx, weight, dweight, bias, dbias, work=B.bload_conv_buffers(pos, x, weight))
        return dx, None, dweight, dbias


class Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, dt, z, b, c, a, d, dt_bias, pos):
        carry, work = B.bload_scan_buffers(pos, x, a, gradient=False, carry=True)
        y = _new(x)
        B.bload_scan(pos, x, dt, a, b, c, y, d, dt_bias, z, carry=carry, work=work)
        ctx.save_for_backward(x, dt, z, b, c, a, d, dt_bias, pos, carry)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, dt, z, b, c, a, d, dt_bias, pos, carry = ctx.saved_tensors
        dx, ddt, dz, db, dc, da, dd, ddt_bias = (_new(v) for v in (x, dt, z, b, c, a, d, dt_bias))
        B.bload_scan_grad(pos, x, dt, a, b, c, carry, dy.contiguous(), dx, ddt, da, db, dc, d, dd, dt_bias, ddt_bias, z, dz,
                          work=B.bload_scan_buffers(pos, x, a, carry=False)[1])
        return dx, ddt, dz, db, dc, da, dd, ddt_bias, None


class RotaryAxes(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, coords, axis, inv_freq):
        ctx.save_for_backward(pos, coords, axis, inv_freq)
        y = _new(x)
        B.bload_rotary_axes(pos, coords, axis, x, y, inv_freq)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        pos, coords, axis, inv_freq = ctx.saved_tensors
        dx = _new(dy)
        B.bload_rotary_axes_grad(pos, coords, axis, dy.contiguous(), dx, inv_freq)
        return dx, None, None, None, None


class Layer(torch.nn.Module):
    def __init__(self, width: int, inner: int, states: int, rank: int = 8, taps: int = 4):
        super().__init__()
        self.inner, self.states, self.rank, self.taps = inner, states, rank, taps
        self.norm_weight, self.norm_bias = torch.nn.Parameter(torch.ones(width)), torch.nn.Parameter(torch.zeros(width))
        self.into = torch.nn.Linear(width, 2 * inner, bias=False)
        self.conv_weight = torch.nn.Parameter(torch.randn(inner, taps) * taps ** -0.5)
        self.conv_bias = torch.nn.Parameter(torch.zeros(inner))
        self.select = torch.nn.Linear(inner, rank + 2 * states, bias=False)
        self.step = torch.nn.Linear(rank, inner, bias=False)
        delta = torch.exp(torch.rand(inner) * 3.0 - 5.0)
        self.dt_bias = torch.nn.Parameter(delta + torch.log(-torch.expm1(-delta)))
        self.log_a = torch.nn.Parameter(torch.log(torch.arange(1, states + 1).float()).repeat(inner, 1))
        self.d = torch.nn.Parameter(torch.ones(inner))
        self.out = torch.nn.Linear(inner, width, bias=False)

    def _selected(self, x):
        """(dt, b, c) of the convolution's output"""
        low, b, c = self.select(x.float()).split((self.rank, self.states, self.states), -1)
        return self.step(low).bfloat16(), b.bfloat16(), c.bfloat16()

    def forward(self, h, pos):
        x, z = self.into(Norm.apply(h, pos, self.norm_weight, self.norm_bias)).bfloat16().chunk(2, -1)
        x = Conv.apply(x, pos, self.conv_weight, self.conv_bias)
        dt, b, c = self._selected(x)
        y = Scan.apply(x, dt, z, b, c, -self.log_a.exp(), self.d, self.dt_bias, pos)
        return h + self.out(y.float())

    @torch.no_grad()
    def prompt(self, h, pos, seq_id, sequences: int):
        """(forward's result, the states behind every sequence)"""
        x, z = self.into(Norm.apply(h, pos, self.norm_weight, self.norm_bias)).bfloat16().chunk(2, -1)
        tails = torch.zeros((sequences, self.taps - 1, self.inner), dtype=x.dtype, device=x.device)
        last = torch.zeros((sequences, self.inner, self.states), device=x.device)
        u, y, a = _new(x), _new(x), -self.log_a.exp()
        B.bload_conv(pos, x, u, self.conv_weight, self.conv_bias, seq_id=seq_id, tails=tails)
        dt, b, c = self._selected(u)
        B.bload_scan(pos, u, dt, a, b, c, y, self.d, self.dt_bias, z, work=B.bload_scan_buffers(pos, u, a, gradient=False)[1], seq_id=seq_id,
                     last=last)
        return h + self.out(y.float()), (tails, last)

    @torch.no_grad()
    def one(self, h, pos, state):
        """The same for one token of each sequence: h [sequences, width], pos [sequences]; the states move on in place."""
        tails, last = state
        n = _new(h)
        B.bload_norm(pos[:, None], h[:, None], n[:, None], self.norm_weight, self.norm_bias)  # (a frame per block)
        x, z = self.into(n).bfloat16().chunk(2, -1)
        u, y = _new(x, x.shape), _new(x, x.shape)
        B.bload_conv_step(pos, tails, x, u, self.conv_weight, self.conv_bias)
        dt, b, c = self._selected(u)
        B.bload_scan_step(pos, last, u, dt, -self.log_a.exp(), b, c, y, self.d, self.dt_bias, z)
        return h + self.out(y.float())


class Model(torch.nn.Module):
    def __init__(self, vocabulary: int, width: int = 96, depth: int = 2, states: int = 16, video: bool = False):
        super().__init__()
        self.embed = torch.nn.Embedding(vocabulary, width)
        self.layers = torch.nn.ModuleList([Layer(width, 2 * width, states) for _ in range(depth)])
        self.head = torch.nn.Linear(width, vocabulary, bias=False)
        self.heads, self.head_dim = 3, 32
        self.video = video
        if video:
            self.qkv = torch.nn.Linear(width, 3 * self.heads * self.head_dim, bias=False)
            self.mix = torch.nn.Linear(self.heads * self.head_dim, width, bias=False)
            n = self.head_dim // 2
            self.register_buffer("inv_freq", 100.0 ** (-torch.arange(n, dtype=torch.float32) / n))
            self.register_buffer("axis", (torch.arange(n) % 2).to(torch.int32))

    def forward(self, tokens, pos):
        h = self.embed(tokens)
        if self.video:
            b, t = tokens.shape
            coords = torch.stack((pos // 4, pos % 4))  # frame and patch
            qkv = self.qkv(h).bfloat16().view(b, t, 3 * self.heads, self.head_dim)
            turned = RotaryAxes.apply(qkv[:, :, :2 * self.heads], pos, coords, self.axis, self.inv_freq)
            a = layers.Attention.apply(turned[:, :, :self.heads], turned[:, :, self.heads:], qkv[:, :, 2 * self.heads:], pos, 0.0)
            h = h + self.mix(a.reshape(b, t, -1).float())
        for layer in self.layers:
            h = layer(h, pos)
        return self.head(h)

    @torch.no_grad()
    def prompt(self, tokens, pos, seq_id, sequences: int):
        h, states = self.embed(tokens), []
        for layer in self.layers:
            h, state = layer.prompt(h, pos, seq_id, sequences)
            states.append(state)
        return self.head(h), states

    @torch.no_grad()
    def one(self, tokens, pos, states):
        h = self.embed(tokens)
        for layer, state in zip(self.layers, states):
            h = layer.one(h, pos, state)
        return self.head(h)


def data(vocabulary: int, t_block: int, device):
    """(lengths, tokens): counting sequences, every token its predecessor plus a stride of the sequence's own"""
    lengths = torch.randint(2, 200, (48,), device=device).clamp_(max=t_block).to(torch.int32)
    starts = lengths.long().cumsum(0) - lengths.long()
    which = torch.repeat_interleave(torch.arange(lengths.numel(), device=device), lengths.long())
    place = torch.arange(int(lengths.sum()), device=device) - starts[which]
    return lengths, (place * (1 + which % 5) + which).remainder(vocabulary).to(torch.int32)


def continue_prompts(model, lengths, tokens, t_block: int, more: int = 4):
    """Continues packed prompts by `more` tokens; (tokens [sequences, more], the largest difference of a step's logits from those
    of the whole sequence in a block of its own, relative to the largest logit)."""
    plan, dense, pos = layers.packed_batch(lengths, tokens, t_block, seed=0)
    seq_id = torch.full_like(pos, -1)
    B.bload_pack(plan, None, 1, 0, plan.n_blocks, seq_id=seq_id)
    n = lengths.numel()
    logits, states = model.prompt(dense, pos, seq_id, n)
    ends = torch.zeros((n, logits.shape[-1]), device=logits.device)
    last = (pos >= 0) & (pos + 1 == lengths[seq_id.clamp(min=0).long()])
    ends[seq_id[last].long()] = logits[last]
    starts = lengths.long().cumsum(0) - lengths.long()
    slots = torch.arange(t_block + more, device=pos.device)[None]
    index = (starts[:, None] + slots).clamp(max=tokens.numel() - 1)
    whole = torch.where(slots < lengths[:, None], tokens[index], 0)
    apart, written = [], []
    for k in range(more):
        token = ends.argmax(-1).to(torch.int32)
        written.append(token)
        at = lengths + k
        whole[torch.arange(n, device=pos.device), at.long()] = token
        ends = model.one(token, at.contiguous(), states)
        alone_pos = torch.where(slots <= at[:, None], slots, -1).to(torch.int32)
        with torch.no_grad():
            want = model(whole, alone_pos)[torch.arange(n, device=pos.device), at.long()]
        apart.append((ends - want).abs().max() / want.abs().max())
    return torch.stack(written, 1), float(torch.stack(apart).max())


def main(steps: int = 40, video: bool = False, device: str = "cuda:0", quiet: bool = False):
    torch.manual_seed(0)
    vocabulary, t_block = 61, 256
    lengths, tokens = data(vocabulary, t_block, device)
    model = Model(vocabulary, video=video).to(device)
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for step in range(steps):
        _, dense, pos = layers.packed_batch(lengths, tokens, t_block, seed=step)
        loss = layers.next_token_loss(model(dense, pos), dense, pos)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
        if not quiet and (step % 10 == 0 or step == steps - 1):
            print("step %3d  loss %.3f" % (step, losses[-1]))
    apart = None
    if not video:
        written, apart = continue_prompts(model, lengths, tokens, t_block)
        if not quiet:
            print("%d prompts continued by %d tokens; a step's logits are within %.2e of those of the whole sequence" % (*written.shape, apart))
    return model, losses, apart


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--video", action="store_true")
    main(**vars(ap.parse_args()))
