"""What the norm, the convolution, the scan and the rotary axes refuse, through the C ABI: every error that the host can see comes
back before the library touches a device, so none is needed here."""
import ctypes as C

import pytest

import paper_2310_10879_b200 as B
from paper_2310_10879_b200 import _lib as E
from test_layers_host import alone

P = 1 << 20  # an address that is never read: the calls below return before that
T = E.ChannelsTensor


def rows(data=P, block=12800, slot=64):
    return T(data, block, slot)


def norm(gradient=False, **change):
    a = E.NormArgs(2, 64, 200, E.BF16, 1e-5, P, P, P, P, rows(), rows(), rows(), rows(), P, P, P, 1 << 40)
    for k, v in change.items():
        setattr(a, k, v)
    L = B.load()
    return (L.bload_norm_grad if gradient else L.bload_norm)(C.byref(a), None)


def common(call):
    assert call(block_count=0) == 0 and call(True, block_count=0) == 0
    assert call(block_count=-1) == E.ERR_ARG and call(t_block=0) == E.ERR_ARG and call(channels=0) == E.ERR_ARG
    assert call(t_block=E.MAX_T_BLOCK + 1) == E.ERR_UNSUPPORTED and call(dtype=3) == E.ERR_UNSUPPORTED and call(dtype=-1) == E.ERR_UNSUPPORTED
    assert call(d_pos=None) == E.ERR_NULL and call(d_pos=P + 2) == E.ERR_ALIGN
    assert call(x=rows(None)) == E.ERR_NULL and call(x=rows(P + 1)) == E.ERR_ALIGN and call(x=rows(slot=-64)) == E.ERR_ARG
    assert call(y=rows(None)) == E.ERR_NULL and call(y=rows(slot=0)) == E.ERR_ARG and call(y=rows(block=0)) == E.ERR_ARG
    assert call(x=rows(block=1 << 40)) == E.ERR_ARG
    assert call(True, dy=rows(None)) == E.ERR_NULL and call(True, dx=rows(slot=0)) == E.ERR_ARG and call(True, dx=rows(P + 1)) == E.ERR_ALIGN
    assert call(True, d_work=None) == E.ERR_NULL and call(True, d_work=P + 16) == E.ERR_ALIGN and call(True, work_bytes=16) == E.ERR_WORKSPACE


def test_norm():
    L = B.load()
    assert L.bload_norm(None, None) == E.ERR_NULL and L.bload_norm_grad(None, None) == E.ERR_NULL
    common(norm)
    assert norm(channels=16385) == E.ERR_UNSUPPORTED and norm(eps=-1.0) == E.ERR_ARG and norm(eps=float("nan")) == E.ERR_ARG
    assert norm(d_weight=P + 2) == E.ERR_ALIGN and norm(d_stats=P + 4) == E.ERR_ALIGN and norm(True, d_dbias=P + 1) == E.ERR_ALIGN
    assert norm(True, d_stats=None) == E.ERR_NULL
    assert L.bload_norm_work_bytes(0, 200, 64, E.BF16) == 0 and L.bload_norm_work_bytes(2, 200, 16385, E.BF16) == 0
    assert L.bload_norm_work_bytes(2, 200, 64, E.BF16) > 0


def conv(gradient=False, **change):
    a = E.ConvArgs(2, 64, 200, E.BF16, 4, 1, P, P, P, rows(), rows(), P, 3, P, rows(), rows(), P, P, P, 1 << 40)
    for k, v in change.items():
        setattr(a, k, v)
    L = B.load()
    return (L.bload_conv_grad if gradient else L.bload_conv)(C.byref(a), None)


def test_conv():
    L = B.load()
    assert L.bload_conv(None, None) == E.ERR_NULL and L.bload_conv_grad(None, None) == E.ERR_NULL
    common(conv)
    assert conv(taps=0) == E.ERR_ARG and conv(taps=9) == E.ERR_UNSUPPORTED and conv(d_weight=None) == E.ERR_NULL
    assert conv(d_weight=P + 2) == E.ERR_ALIGN and conv(d_bias=P + 1) == E.ERR_ALIGN and conv(True, d_dweight=P + 2) == E.ERR_ALIGN
    assert conv(d_seq_id=None) == E.ERR_NULL and conv(n_seq=-1) == E.ERR_ARG and conv(d_tails=P + 1) == E.ERR_ALIGN
    assert conv(channels=1 << 31) == E.ERR_ARG and conv(block_count=1 << 30, channels=4096) == E.ERR_ARG
    assert L.bload_conv_work_bytes(1 << 30, 200, 4096, 4, E.BF16) == 0 and L.bload_conv_work_bytes(2, 200, 64, 9, E.BF16) == 0


def conv_step(n=4, c=64, dtype=E.BF16, taps=4, pos=P, state=P, after=P, x=rows(), y=rows(), w=P, bias=P):
    return B.load().bload_conv_step(n, c, dtype, taps, 1, pos, state, after, x and C.byref(x), y and C.byref(y), w, bias, None)


def test_conv_step():
    assert conv_step(n=0) == 0
    assert conv_step(n=-1) == E.ERR_ARG and conv_step(c=0) == E.ERR_ARG and conv_step(n=1 << 40) == E.ERR_ARG and conv_step(taps=0) == E.ERR_ARG
    assert conv_step(taps=9) == E.ERR_UNSUPPORTED and conv_step(dtype=5) == E.ERR_UNSUPPORTED
    for name in ("pos", "state", "after", "x", "y", "w"):
        assert conv_step(**{name: None}) == E.ERR_NULL, name
    assert conv_step(x=rows(None)) == E.ERR_NULL and conv_step(y=rows(block=0)) == E.ERR_ARG and conv_step(x=rows(block=-1)) == E.ERR_ARG
    assert conv_step(state=P + 1) == E.ERR_ALIGN and conv_step(pos=P + 2) == E.ERR_ALIGN and conv_step(bias=P + 2) == E.ERR_ALIGN


def scan(gradient=False, **change):
    a = E.ScanArgs(2, 64, 200, E.BF16, 16, 1, P, P, P, P, *[rows() for _ in range(6)], P, P, 1 << 40, P, 3, P, *[rows() for _ in range(6)], P, P, P)
    for k, v in change.items():
        setattr(a, k, v)
    L = B.load()
    return (L.bload_scan_grad if gradient else L.bload_scan)(C.byref(a), None)


def test_scan():
    L = B.load()
    assert L.bload_scan(None, None) == E.ERR_NULL and L.bload_scan_grad(None, None) == E.ERR_NULL
    common(scan)
    assert scan(states=0) == E.ERR_ARG and scan(states=65) == E.ERR_UNSUPPORTED
    for name in ("dt", "b", "c"):
        assert scan(**{name: rows(None)}) == E.ERR_NULL and scan(**{name: rows(P + 1)}) == E.ERR_ALIGN, name
    assert scan(z=rows(P + 1)) == E.ERR_ALIGN and scan(z=rows(slot=-1)) == E.ERR_ARG
    assert scan(d_a=None) == E.ERR_NULL and scan(d_a=P + 2) == E.ERR_ALIGN and scan(d_carry=P + 8) == E.ERR_ALIGN
    assert scan(d_seq_id=None) == E.ERR_NULL and scan(n_seq=-1) == E.ERR_ARG and scan(d_last=P + 2) == E.ERR_ALIGN
    assert scan(True, d_carry=None) == E.ERR_NULL and scan(True, d_da=None) == E.ERR_NULL and scan(True, dz=rows(None)) == E.ERR_NULL
    assert scan(True, db=rows(slot=0)) == E.ERR_ARG and scan(True, ddt=rows(None)) == E.ERR_NULL and scan(True, d_dd=P + 1) == E.ERR_ALIGN


def scan_step(**change):
    a = E.ScanStepArgs(4, 64, E.BF16, 16, 1, P, P, P, P, P, P, *[rows() for _ in range(6)])
    for k, v in change.items():
        setattr(a, k, v)
    return B.load().bload_scan_step(C.byref(a), None)


def test_scan_step():
    assert B.load().bload_scan_step(None, None) == E.ERR_NULL
    assert scan_step(rows=0) == 0
    assert scan_step(rows=-1) == E.ERR_ARG and scan_step(rows=1 << 40) == E.ERR_ARG and scan_step(channels=0) == E.ERR_ARG
    assert scan_step(states=0) == E.ERR_ARG and scan_step(states=65) == E.ERR_UNSUPPORTED and scan_step(dtype=3) == E.ERR_UNSUPPORTED
    for name in ("d_pos", "d_a", "state", "next"):
        assert scan_step(**{name: None}) == E.ERR_NULL, name
    for name in ("x", "dt", "b", "c", "y"):
        assert scan_step(**{name: rows(None)}) == E.ERR_NULL, name
    assert scan_step(y=rows(block=0)) == E.ERR_ARG and scan_step(state=P + 2) == E.ERR_ALIGN and scan_step(z=rows(P + 1)) == E.ERR_ALIGN


def axes(pos=P, coords=P, n=3, axis=P, b=2, x=E.HeadsTensor(P, 16384, 256, 64), y=E.HeadsTensor(P, 16384, 256, 64), rot=64):
    L = B.load()
    got = {fn(pos, coords, n, axis, b, 64, 4, 64, E.BF16, C.byref(x), C.byref(y), P, rot, 0, 1.0, None)
           for fn in (L.bload_rotary_axes, L.bload_rotary_axes_grad)}
    assert len(got) == 1
    return got.pop()


def test_rotary_axes():
    assert axes(b=0) == 0
    assert axes(n=0) == E.ERR_ARG and axes(n=5) == E.ERR_ARG and axes(rot=66) == E.ERR_ARG and axes(b=-1) == E.ERR_ARG
    assert axes(pos=None) == E.ERR_NULL and axes(coords=None) == E.ERR_NULL and axes(axis=None) == E.ERR_NULL
    assert axes(coords=P + 2) == E.ERR_ALIGN and axes(axis=P + 1) == E.ERR_ALIGN


def test_the_packed_argument_blocks_have_the_layout_of_the_structures():

    n = E.NormArgs.from_buffer_copy(E._NORM.pack(1, 2, 3, 4, 0.5, *range(10, 30)))
    assert (n.block_count, n.channels, n.t_block, n.dtype, n.eps, n.d_pos, n.d_stats, n.x.data, n.dx.slot_stride) == (1, 2, 3, 4, 0.5, 10, 13, 14, 25)
    assert (n.d_dweight, n.work_bytes) == (26, 29)
    c = E.ConvArgs.from_buffer_copy(E._CONV.pack(*range(1, 29)))
    assert (c.taps, c.silu, c.d_pos, c.x.data, c.y.slot_stride, c.d_seq_id, c.n_seq, c.d_tails, c.dy.data, c.d_dweight, c.work_bytes) == (
        5, 6, 7, 10, 15, 16, 17, 18, 19, 25, 28)
    s = E.ScanArgs.from_buffer_copy(E._SCAN.pack(*range(1, 56)))
    assert (s.states, s.softplus, s.d_pos, s.d_dt_bias, s.x.data, s.y.slot_stride, s.d_carry, s.work_bytes, s.d_seq_id, s.d_last) == (
        5, 6, 7, 10, 11, 28, 29, 31, 32, 34)
    assert (s.dy.data, s.dz.slot_stride, s.d_da, s.d_ddt_bias) == (35, 52, 53, 55)
    p = E.ScanStepArgs.from_buffer_copy(E._SCAN_STEP.pack(*range(1, 30)))
    assert (p.softplus, p.d_pos, p.state, p.next, p.x.data, p.y.slot_stride) == (5, 6, 10, 11, 12, 29)
    for packed, structure in ((E._NORM, E.NormArgs), (E._CONV, E.ConvArgs), (E._SCAN, E.ScanArgs), (E._SCAN_STEP, E.ScanStepArgs), (E._CHANNELS, T)):
        assert packed.size == C.sizeof(structure)


SIZES_WITHOUT_END = """
from paper_2310_10879_b200 import _lib as E
L, P = E.load(), 1 << 20
sizes = (1, 2, 63, 4096, (1 << 31) - 1, 1 << 31, 1 << 40, 1 << 58, (1 << 62) + 1, (1 << 63) - 1)
for blocks in sizes:
    for t in (1, 64, 5000, E.MAX_T_BLOCK):
        for channels in sizes:
            for states in (1, 16, 64):
                ok = blocks < 1 << 31 and channels < 1 << 31
                # Python's integers have no end
                fits = ok and blocks * (channels // 16 + 1) < 1 << 31 and blocks * t <= 1 << 31 and blocks * channels * (states + 2) <= 1 << 35
                for gradient in (0, 1):
                    need = L.bload_scan_work_bytes(blocks, t, channels, states, gradient)
                    assert need < 1 << 52 and (fits or need == 0) and (not fits or not gradient or need > 0), (blocks, t, channels, states, need)
            fits = ok and blocks * -(-t // 32) * (channels // 256 + 1) < 1 << 31
            need = L.bload_conv_work_bytes(blocks, t, channels, 4, E.F32)
            assert need < 1 << 52 and (need > 0) == fits, (blocks, t, channels, need)
            need = L.bload_norm_work_bytes(blocks, t, channels, E.F32)
            assert need < 1 << 40 and (need > 0) == (blocks < 1 << 31 and channels <= 16384)
"""


def test_sizes_whose_product_has_no_room_are_refused():
    assert alone(SIZES_WITHOUT_END) == 0


NO_DEVICE = """
from paper_2310_10879_b200 import _lib as E
import ctypes as C
L, P = E.load(), 1 << 20
rows = lambda: E.ChannelsTensor(P, 12800, 64)
n = E.NormArgs(2, 64, 200, E.BF16, 1e-5, P, P, P, P, rows(), rows(), rows(), rows(), P, P, P, 1 << 40)
c = E.ConvArgs(2, 64, 200, E.BF16, 4, 1, P, P, P, rows(), rows(), P, 3, P, rows(), rows(), P, P, P, 1 << 40)
s = E.ScanArgs(2, 64, 200, E.BF16, 16, 1, P, P, P, P, *[rows() for _ in range(6)], P, P, 1 << 40, P, 3, P, *[rows() for _ in range(6)], P, P, P)
p = E.ScanStepArgs(4, 64, E.BF16, 16, 1, P, P, P, P, P, P, *[rows() for _ in range(6)])
for call, a in ((L.bload_norm, n), (L.bload_norm_grad, n), (L.bload_conv, c), (L.bload_conv_grad, c), (L.bload_scan, s), (L.bload_scan_grad, s),
                (L.bload_scan_step, p)):
    rc = call(C.byref(a), None)
    assert rc == E.ERR_CUDA, (call, rc)  # every argument was taken, and there is no device
x = rows()
assert L.bload_conv_step(4, 64, E.BF16, 4, 1, P, P, P, C.byref(x), C.byref(x), P, P, None) == E.ERR_CUDA
h = E.HeadsTensor(P, 16384, 256, 64)
assert L.bload_rotary_axes(P, P, 3, P, 2, 64, 4, 64, E.BF16, C.byref(h), C.byref(h), P, 64, 0, 1.0, None) == E.ERR_CUDA
"""


def test_a_missing_device_is_an_error_and_nothing_worse():
    assert alone(NO_DEVICE) == 0
