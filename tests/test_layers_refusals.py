"""What the layers on packed batches refuse, through the C ABI: every error that the host can see comes back before the
library touches a device, so none is needed here."""
import ctypes as C

import paper_2310_10879_b200 as B
from paper_2310_10879_b200 import _lib as E

P = 1 << 20  # an address that is never read: the calls below return before that


def heads(data=P, block=64 * 4 * 64, slot=4 * 64, head=64):
    return E.HeadsTensor(data, block, slot, head)


def attention(gradient=False, **change):
    a = E.AttentionArgs(2, 64, 4, 4, 64, E.BF16, 1, 0, 0.125, 0.0, P, None)
    for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        setattr(a, n, heads())
    a.d_lse, a.d_delta = P, P
    for k, v in change.items():
        setattr(a, k, v)
    L = B.load()
    return (L.bload_attention_grad if gradient else L.bload_attention)(C.byref(a), None)


def test_attention():
    L = B.load()
    assert L.bload_attention(None, None) == E.ERR_NULL and L.bload_attention_grad(None, None) == E.ERR_NULL
    assert attention(block_count=0) == 0 and attention(True, block_count=0) == 0
    assert attention(block_count=-1) == E.ERR_ARG and attention(t_block=0) == E.ERR_ARG
    assert attention(t_block=E.MAX_T_BLOCK + 1) == E.ERR_UNSUPPORTED
    assert attention(heads=0) == E.ERR_ARG and attention(kv_heads=0) == E.ERR_ARG and attention(kv_heads=3) == E.ERR_ARG
    assert attention(head_dim=0) == E.ERR_ARG and attention(head_dim=60) == E.ERR_UNSUPPORTED
    assert attention(head_dim=136) == E.ERR_UNSUPPORTED
    assert attention(dtype=E.F32) == E.ERR_UNSUPPORTED and attention(dtype=3) == E.ERR_UNSUPPORTED
    assert attention(window=-1) == E.ERR_ARG and attention(softcap=-1.0) == E.ERR_ARG
    assert attention(softcap=float("inf")) == E.ERR_ARG and attention(scale=float("nan")) == E.ERR_ARG
    assert attention(d_pos=None) == E.ERR_NULL and attention(d_pos=P + 2) == E.ERR_ALIGN
    assert attention(q=heads(None)) == E.ERR_NULL and attention(v=heads(P + 8)) == E.ERR_ALIGN
    assert attention(k=heads(slot=0)) == E.ERR_ARG and attention(out=heads(head=-64)) == E.ERR_ARG
    assert attention(k=heads(slot=260)) == E.ERR_ALIGN and attention(out=heads(block=1 << 40)) == E.ERR_ARG
    assert attention(d_lse=P + 2) == E.ERR_ALIGN and attention(d_slopes=P + 1) == E.ERR_ALIGN
    assert attention(True, d_lse=None) == E.ERR_NULL and attention(True, d_delta=None) == E.ERR_NULL
    assert attention(True, dk=heads(None)) == E.ERR_NULL and attention(True, dq=heads(P + 4)) == E.ERR_ALIGN


def recurrence(gradient=False, **change):
    a = E.RecurrenceArgs(2, 64, 200, E.BF16, P)
    for n in ("gate", "x", "h", "dh", "dgate", "dx"):
        setattr(a, n, E.ChannelsTensor(P, 200 * 64, 64))
    a.d_carry, a.d_work, a.work_bytes = P, P, 1 << 40
    for k, v in change.items():
        setattr(a, k, v)
    L = B.load()
    return (L.bload_recurrence_grad if gradient else L.bload_recurrence)(C.byref(a), None)


def test_recurrence():
    L = B.load()
    T = E.ChannelsTensor
    assert L.bload_recurrence(None, None) == E.ERR_NULL and L.bload_recurrence_grad(None, None) == E.ERR_NULL
    assert recurrence(block_count=0) == 0 and recurrence(True, block_count=0) == 0
    assert recurrence(block_count=-1) == E.ERR_ARG and recurrence(t_block=0) == E.ERR_ARG and recurrence(channels=0) == E.ERR_ARG
    assert recurrence(t_block=E.MAX_T_BLOCK + 1) == E.ERR_UNSUPPORTED and recurrence(dtype=7) == E.ERR_UNSUPPORTED
    assert recurrence(d_pos=None) == E.ERR_NULL and recurrence(gate=T(None, 12800, 64)) == E.ERR_NULL
    assert recurrence(x=T(P + 1, 12800, 64)) == E.ERR_ALIGN and recurrence(x=T(P, 12800, -64)) == E.ERR_ARG
    assert recurrence(h=T(P, 12800, 0)) == E.ERR_ARG and recurrence(d_carry=P + 4) == E.ERR_ALIGN
    assert recurrence(True, d_carry=None) == E.ERR_NULL and recurrence(True, dx=T(P, 0, 64)) == E.ERR_ARG


def rotary(pos=P, b=2, t=64, h=4, d=64, dtype=E.BF16, x=heads(), y=heads(), inv=P, rot=64, factor=1.0):
    L = B.load()
    got = {fn(pos, b, t, h, d, dtype, x and C.byref(x), y and C.byref(y), inv, rot, 0, factor, None)
           for fn in (L.bload_rotary, L.bload_rotary_grad)}
    assert len(got) == 1
    return got.pop()


def test_rotary():
    assert rotary(b=0) == 0
    assert rotary(pos=None) == E.ERR_NULL and rotary(x=None) == E.ERR_NULL and rotary(y=None) == E.ERR_NULL
    assert rotary(inv=None) == E.ERR_NULL and rotary(inv=P + 2) == E.ERR_ALIGN
    assert rotary(b=-1) == E.ERR_ARG and rotary(t=0) == E.ERR_ARG and rotary(h=0) == E.ERR_ARG and rotary(d=0) == E.ERR_ARG
    assert rotary(rot=63) == E.ERR_ARG and rotary(rot=66) == E.ERR_ARG and rotary(rot=-2) == E.ERR_ARG
    assert rotary(dtype=-1) == E.ERR_UNSUPPORTED and rotary(t=E.MAX_T_BLOCK + 1) == E.ERR_UNSUPPORTED
    assert rotary(factor=float("nan")) == E.ERR_ARG
    assert rotary(x=heads(P + 1)) == E.ERR_ALIGN and rotary(y=heads(head=0)) == E.ERR_ARG and rotary(x=heads(slot=-1)) == E.ERR_ARG


def test_the_packed_argument_blocks_have_the_layout_of_the_structures():
    assert E._HEADS.size == C.sizeof(E.HeadsTensor)
    assert E._ATTENTION_GRAD.size == C.sizeof(E.AttentionArgs) and E._RECURRENCE.size == C.sizeof(E.RecurrenceArgs)
    a = E.AttentionArgs.from_buffer_copy(E._ATTENTION_GRAD.pack(*range(1, 9), 0.5, 0.25, 0, *range(20, 56)))
    assert (a.block_count, a.t_block, a.heads, a.kv_heads, a.head_dim, a.dtype, a.causal, a.window) == tuple(range(1, 9))
    assert (a.scale, a.softcap, a.d_pos, a.d_slopes, a.q.data, a.q.head_stride, a.out.data, a.d_lse) == (0.5, 0.25, 20, 21, 22, 25, 34, 38)
    assert (a.dout.data, a.dv.head_stride, a.d_delta) == (39, 54, 55)
    assert E._ATTENTION.size == E.AttentionArgs.d_lse.offset + 8
    r = E.RecurrenceArgs.from_buffer_copy(E._RECURRENCE.pack(*range(1, 27)))
    assert (r.block_count, r.channels, r.t_block, r.dtype, r.d_pos, r.gate.data, r.h.slot_stride) == (1, 2, 3, 4, 5, 6, 14)
    assert (r.d_carry, r.d_work, r.work_bytes, r.dh.data, r.dx.slot_stride) == (15, 16, 17, 18, 26)
