"""A small sequence model trained on packed blocks: rotary attention and a gated recurrence, both of which read the
per-slot positions that bload_pack writes and stay inside sequences.

    python examples/packed_layers.py [--steps N]

Per batch: plan and pack token ids with their positions, embed, mix along the slots with both layers, predict the next
token of the same sequence, and take a gradient step.  Beside the loss it reports how far the packed batch's outputs are
from those of every sequence in a block of its own, which is how far a sequence is from noticing its neighbours.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2310_10879_b200 as B  # noqa: E402


class Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, pos, inv_freq):
        ctx.save_for_backward(pos, inv_freq)
        y = torch.empty_like(x)
        B.bload_rotary(pos, x, y, inv_freq)
        return y

    @staticmethod
    @once_differentiable  # (the gradient calls have no gradients of their own)
    def backward(ctx, dy):
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        B.bload_rotary_grad(ctx.saved_tensors[0], dy.contiguous(), dx, ctx.saved_tensors[1])
        return dx, None, None


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, pos, softcap):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
        B.bload_attention(pos, q, k, v, out, lse, softcap=softcap)
        ctx.save_for_backward(q, k, v, pos, out, lse)
        ctx.softcap = softcap
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, pos, out, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v))
        B.bload_attention_grad(pos, q, k, v, out, lse, dout.contiguous(), dq, dk, dv, torch.empty_like(lse), softcap=ctx.softcap)
        return dq, dk, dv, None, None


class Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, x, pos):
        carry, work = B.bload_recurrence_buffers(pos, x)
        h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        B.bload_recurrence(pos, gate, x, h, carry, work)
        ctx.save_for_backward(gate, x, pos, carry)
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dh):
        gate, x, pos, carry = ctx.saved_tensors
        dgate, dx = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for _ in range(2))
        work = B.bload_recurrence_buffers(pos, x)[1]
        B.bload_recurrence_grad(pos, gate, x, carry, dh.contiguous(), dgate, dx, work)
        return dgate, dx, None


class Model(torch.nn.Module):
    def __init__(self, vocabulary: int, width: int = 128, heads: int = 4, kv_heads: int = 2, head_dim: int = 32):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.embed = torch.nn.Embedding(vocabulary, width)
        self.qkv = torch.nn.Linear(width, (heads + 2 * kv_heads) * head_dim, bias=False)
        self.out = torch.nn.Linear(heads * head_dim, width, bias=False)
        self.gate_x = torch.nn.Linear(width, 2 * width)
        self.norms = torch.nn.ModuleList([torch.nn.LayerNorm(width) for _ in range(3)])
        self.head = torch.nn.Linear(width, vocabulary, bias=False)
        n = head_dim // 2
        self.register_buffer("inv_freq", 10000.0 ** (-torch.arange(n, dtype=torch.float32) / n))

    def forward(self, tokens, pos):
        b, t = tokens.shape
        x = self.embed(tokens)
        qkv = self.qkv(self.norms[0](x)).bfloat16().view(b, t, self.heads + 2 * self.kv_heads, self.head_dim)
        turned = Rotary.apply(qkv[:, :, :self.heads + self.kv_heads], pos, self.inv_freq)  # queries and keys in one call
        a = Attention.apply(turned[:, :, :self.heads], turned[:, :, self.heads:], qkv[:, :, self.heads + self.kv_heads:], pos, 30.0)
        x = x + self.out(a.reshape(b, t, -1).float())
        gate, into = self.gate_x(self.norms[1](x)).bfloat16().chunk(2, -1)
        x = x + Recurrence.apply(gate, into, pos).float()
        return self.head(self.norms[2](x))


def packed_batch(lengths, tokens, t_block: int, seed: int):
    """(token ids, positions) of every block of a plan, both int32 [blocks, t_block]."""
    plan = B.bload_plan(lengths, t_block, seed)
    shape = (plan.n_blocks, t_block)
    dense = torch.empty(shape, dtype=torch.int32, device=tokens.device)
    pos = torch.empty(shape, dtype=torch.int32, device=tokens.device)
    B.bload_pack(plan, tokens, 4, 0, plan.n_blocks, dense=dense, pos=pos)
    return plan, dense, pos


def next_token_loss(logits, tokens, pos):
    follows = pos[:, 1:] > 0  # the slot's token belongs to the same sequence as the one before it
    return torch.nn.functional.cross_entropy(logits[:, :-1][follows], tokens[:, 1:][follows].long())


def main(steps: int = 40, device: str = "cuda:0", quiet: bool = False):
    torch.manual_seed(0)
    vocabulary, t_block = 61, 256
    lengths = torch.randint(2, 200, (48,), device=device).clamp_(max=t_block).to(torch.int32)
    total = int(lengths.sum())
    # counting sequences: every token is its predecessor plus a stride of the sequence's own
    starts = lengths.long().cumsum(0) - lengths.long()
    which = torch.repeat_interleave(torch.arange(lengths.numel(), device=device), lengths.long())
    tokens = ((torch.arange(total, device=device) - starts[which]) * (1 + which % 5) + which).remainder(vocabulary).to(torch.int32)
    model = Model(vocabulary).to(device)
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    losses = []
    for step in range(steps):
        _, dense, pos = packed_batch(lengths, tokens, t_block, seed=step)
        loss = next_token_loss(model(dense, pos), dense, pos)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
        if not quiet and (step % 10 == 0 or step == steps - 1):
            print("step %3d  loss %.3f" % (step, losses[-1]))
    # every sequence in a block of its own: the same logits, up to the rounding of another order of sums
    plan, dense, pos = packed_batch(lengths, tokens, t_block, seed=0)
    alone = torch.arange(t_block, device=device, dtype=torch.int32)[None].repeat(lengths.numel(), 1)
    alone_pos = torch.where(alone < lengths[:, None], alone, -1)
    index = (starts[:, None] + alone.long()).clamp_(max=total - 1)
    with torch.no_grad():
        packed, single = model(dense, pos), model(tokens[index].where(alone_pos >= 0, torch.zeros_like(alone)), alone_pos)
    tables = plan.tables()
    seq_id = torch.full_like(pos, -1)
    B.bload_pack(plan, None, 1, 0, plan.n_blocks, seq_id=seq_id)
    frame = pos >= 0
    apart = (packed[frame] - single[seq_id[frame].long(), pos[frame].long()]).abs().max() / packed[frame].abs().max()
    if not quiet:
        print("blocks %d, sequences %d, largest difference from sequences on their own %.2e of the largest logit" % (
            plan.n_blocks, tables["seg_seq"].numel(), float(apart)))
    return losses, float(apart)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=40)
    main(ap.parse_args().steps)
