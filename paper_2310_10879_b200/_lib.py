"""ctypes binding of libbload.so: argument marshalling only.

Every step of the path runs inside the library's CUDA kernels; torch is used for device memory
and streams.  There is no CPU fallback: if the shared library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("BLOAD_LIBRARY") or os.path.join(_HERE, "libbload.so")  # override: a build to compare

OK = 0
ERR_NULL, ERR_ARG, ERR_LENGTH, ERR_WORKSPACE, ERR_ALIGN = -1, -2, -3, -4, -5
ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT, ERR_PLAN = -6, -7, -8, -9
MAX_T_BLOCK = 32768

EXPORTS = ("bload_plan_sizes", "bload_plan", "bload_plan_async", "bload_plan_finish", "bload_rank_range", "bload_pack", "bload_unpack", "bload_stats", "bload_epoch", "bload_epoch_stage_times",
           "bload_pack_repeat_last", "bload_var_offsets", "bload_pack_var", "bload_unpack_var", "bload_var_offsets2d", "bload_pack_var2d",
           "bload_unpack_var2d", "bload_carry_prev", "bload_reset_state", "bload_valid_sum",
           "bload_rotary", "bload_rotary_grad", "bload_attention", "bload_attention_grad", "bload_recurrence_work_bytes",
           "bload_recurrence", "bload_recurrence_grad", "bload_device_timeouts",
           "bload_rotary_axes", "bload_rotary_axes_grad", "bload_norm_work_bytes", "bload_norm", "bload_norm_grad",
           "bload_conv_work_bytes", "bload_conv", "bload_conv_grad", "bload_conv_step",
           "bload_scan_work_bytes", "bload_scan", "bload_scan_grad", "bload_scan_step",
           "bload_plan_static", "bload_chunk_work_bytes", "bload_chunk_count", "bload_plan_chunks", "bload_set_plan_timing", "bload_plan_stage_times", "bload_kernel_launches", "bload_last_copy_kernel", "bload_debug_status", "bload_bulk_copy_timeouts",
           "bload_strerror", "bload_version")


class Sizes(C.Structure):
    _fields_ = [("plan_bytes", C.c_size_t), ("work_bytes", C.c_size_t), ("max_blocks", C.c_int64)] + \
               [(k, C.c_size_t) for k in ("off_offsets", "off_seg_seq", "off_seg_block", "off_seg_start",
                                          "off_seg_src", "off_block_seg_begin", "off_block_fill",
                                          "off_seq_block", "off_seq_start")]


class PlanInfo(C.Structure):
    _fields_ = [("status", C.c_int32), ("t_block", C.c_int32), ("n", C.c_int64), ("n_blocks", C.c_int64),
                ("sum_t", C.c_int64), ("t_max", C.c_int64), ("first_bad_index", C.c_int64),
                ("checksum", C.c_uint64), ("max_segs_per_block", C.c_int64), ("seed", C.c_uint64),
                ("policy", C.c_uint32), ("n_source", C.c_uint32)]


class Stats(C.Structure):
    _fields_ = [(k, C.c_int64) for k in ("n", "sum_t", "t_max", "t_block", "n_blocks", "pad_packed",
                                          "pad_naive_tmax", "pad_naive_tblock", "min_blocks")] + \
               [(k, C.c_double) for k in ("frac_packed", "frac_naive_tmax", "frac_naive_tblock",
                                          "reduction_vs_tmax", "mean_segs_per_block")] + \
               [("max_segs_per_block", C.c_int64), ("frames_deleted", C.c_int64)]


class EpochIO(C.Structure):
    _fields_ = [("d_store", C.c_void_p), ("frame_bytes", C.c_int64), ("d_dense", C.c_void_p),
                ("d_seq_id", C.c_void_p), ("d_pos", C.c_void_p), ("d_reset", C.c_void_p), ("d_valid", C.c_void_p),
                ("d_dense_out", C.c_void_p), ("out_frame_bytes", C.c_int64), ("d_ragged_out", C.c_void_p),
                ("block_capacity", C.c_int64), ("pad_byte", C.c_uint8), ("chunks", C.c_uint8), ("reserved_", C.c_uint8 * 6)]


class ChunkInfo(C.Structure):
    _fields_ = [("status", C.c_int32), ("tail", C.c_uint32), ("t_chunk", C.c_int32), ("reserved_", C.c_int32)] + \
               [(k, C.c_int64) for k in ("n", "n_chunks", "frames_kept", "frames_deleted", "pad_frames", "sum_t", "t_max",
                                          "first_bad_index")]


class VarInfo(C.Structure):
    _fields_ = [("total_bytes", C.c_int64), ("max_frame_bytes", C.c_int64), ("first_bad_index", C.c_int64),
                ("max_rows", C.c_int64)]


class BloadError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (%d)" % (where, strerror(code), code))


_lib = None


def load() -> C.CDLL:
    """Load libbload.so.  Raises if it has not been built (python -m paper_2310_10879_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if "BLOAD_LIBRARY" not in os.environ:
        # a missing or stale in-tree library is (re)built from the CUDA sources; if that is impossible, fail loudly:
        # a library built from other sources than the ones in this tree must never run unnoticed
        from . import build as _build
        try:
            _build.build()
        except Exception as exc:
            what = "is missing" if not os.path.exists(LIB_PATH) else "was built from other sources than this tree's"
            raise RuntimeError("libbload.so at %s %s and could not be rebuilt (%s); there is no CPU fallback.  Build it "
                               "with `python -m paper_2310_10879_b200.build`, or name a library to load with "
                               "BLOAD_LIBRARY" % (LIB_PATH, what, exc)) from exc
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libbload.so is missing at %s: build it with `python -m paper_2310_10879_b200.build` "
                           "(there is no CPU fallback)" % LIB_PATH)
    L = C.CDLL(LIB_PATH)
    vp, i64, i32, u64, u32, u8 = C.c_void_p, C.c_int64, C.c_int32, C.c_uint64, C.c_uint32, C.c_uint8
    L.bload_plan_sizes.argtypes = [i64, i32, C.POINTER(Sizes)]
    L.bload_plan.argtypes = [vp, i64, i32, u64, u32, vp, C.c_size_t, vp, C.c_size_t, vp, C.POINTER(PlanInfo)]
    L.bload_plan_async.argtypes = [vp, i64, i32, u64, u32, vp, C.c_size_t, vp, C.c_size_t, vp]
    L.bload_chunk_work_bytes.argtypes = [i64]
    L.bload_chunk_count.argtypes = [vp, i64, i32, u32, vp, C.c_size_t, vp, C.POINTER(ChunkInfo)]
    L.bload_plan_chunks.argtypes = [vp, i64, i32, u32, i64, vp, C.c_size_t, vp, C.c_size_t, vp, vp, vp, C.POINTER(PlanInfo)]
    L.bload_plan_static.argtypes = [vp, i64, i32, u64, u32, vp, C.c_size_t, vp, C.POINTER(PlanInfo)]
    L.bload_plan_finish.argtypes = [vp, vp, C.POINTER(PlanInfo)]
    L.bload_rank_range.argtypes = [i64, i32, i32, i32, C.POINTER(i64), C.POINTER(i64)]
    L.bload_pack.argtypes = [vp, C.POINTER(PlanInfo), vp, i64, i64, i64, vp, vp, vp, vp, vp, u8, vp]
    L.bload_pack_repeat_last.argtypes = L.bload_pack.argtypes
    L.bload_unpack.argtypes = [vp, C.POINTER(PlanInfo), vp, i64, i64, i64, vp, vp]
    L.bload_stats.argtypes = [C.POINTER(PlanInfo), C.POINTER(Stats)]
    L.bload_var_offsets.argtypes = [vp, vp, i64, vp, vp, C.POINTER(VarInfo)]
    L.bload_pack_var.argtypes = [vp, C.POINTER(PlanInfo), vp, vp, vp, i64, i64, i64, vp, u8, vp]
    L.bload_unpack_var.argtypes = [vp, C.POINTER(PlanInfo), vp, vp, vp, i64, i64, i64, vp, vp]
    L.bload_var_offsets2d.argtypes = [vp, vp, vp, i64, vp, vp, C.POINTER(VarInfo)]
    L.bload_pack_var2d.argtypes = [vp, C.POINTER(PlanInfo), vp, vp, vp, vp, i64, i64, i64, i64, vp, u8, vp]
    L.bload_unpack_var2d.argtypes = [vp, C.POINTER(PlanInfo), vp, vp, vp, vp, i64, i64, i64, i64, vp, vp]
    L.bload_carry_prev.argtypes = [vp, C.POINTER(PlanInfo), vp, i64, i64, i64, vp, u8, vp]
    L.bload_reset_state.argtypes = [vp, C.POINTER(PlanInfo), i64, i64, i32, vp, i64, vp, vp]
    L.bload_valid_sum.argtypes = [vp, C.POINTER(PlanInfo), vp, i64, i64, vp, vp, vp]
    L.bload_epoch.argtypes = [vp, i64, i32, u64, vp, C.c_size_t, vp, C.c_size_t, C.POINTER(EpochIO), vp, vp,
                              C.POINTER(PlanInfo)]
    L.bload_epoch_stage_times.argtypes = [C.POINTER(C.c_float * 5)]
    L.bload_rotary.argtypes = [vp, i64, i32, i32, i32, i32, vp, vp, vp, i32, i32, C.c_float, vp]
    L.bload_rotary_grad.argtypes = L.bload_rotary.argtypes
    L.bload_attention.argtypes = [vp, vp]
    L.bload_attention_grad.argtypes = L.bload_attention.argtypes
    L.bload_recurrence_work_bytes.argtypes = [i64, i32, i64]
    L.bload_recurrence.argtypes = [vp, vp]
    L.bload_recurrence_grad.argtypes = L.bload_recurrence.argtypes
    L.bload_rotary_axes.argtypes = [vp, vp, i32, vp, i64, i32, i32, i32, i32, vp, vp, vp, i32, i32, C.c_float, vp]
    L.bload_rotary_axes_grad.argtypes = L.bload_rotary_axes.argtypes
    L.bload_norm_work_bytes.argtypes = [i64, i32, i64, i32]
    L.bload_conv_work_bytes.argtypes = [i64, i32, i64, i32, i32]
    L.bload_scan_work_bytes.argtypes = [i64, i32, i64, i32, i32]
    for name in ("bload_norm", "bload_norm_grad", "bload_conv", "bload_conv_grad", "bload_scan", "bload_scan_grad", "bload_scan_step"):
        getattr(L, name).argtypes = [vp, vp]
    L.bload_conv_step.argtypes = [i64, i64, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    L.bload_set_plan_timing.argtypes = [C.c_int]
    L.bload_plan_stage_times.argtypes = [C.POINTER(C.c_float * 4)]
    L.bload_strerror.argtypes = [C.c_int]
    L.bload_strerror.restype = C.c_char_p
    L.bload_last_copy_kernel.argtypes = [C.c_int]
    L.bload_debug_status.argtypes = [C.POINTER(C.c_uint64 * 4), C.c_int]
    L.bload_version.argtypes = []
    L.bload_kernel_launches.argtypes = []
    for name in EXPORTS:
        if name not in ("bload_strerror", "bload_kernel_launches", "bload_last_copy_kernel", "bload_debug_status", "bload_bulk_copy_timeouts", "bload_device_timeouts") and not name.endswith("_work_bytes"):
            getattr(L, name).restype = C.c_int
    L.bload_kernel_launches.restype = C.c_int64
    L.bload_device_timeouts.argtypes = []
    L.bload_device_timeouts.restype = C.c_int64
    L.bload_bulk_copy_timeouts.argtypes = []
    L.bload_bulk_copy_timeouts.restype = C.c_int64
    L.bload_chunk_work_bytes.restype = C.c_size_t
    for name in ("recurrence", "norm", "conv", "scan"):
        getattr(L, "bload_%s_work_bytes" % name).restype = C.c_size_t
    L.bload_last_copy_kernel.restype = C.c_char_p
    _lib = L
    return L


def strerror(code: int) -> str:
    return load().bload_strerror(code).decode()


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def _stream(stream) -> int | None:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


def bload_plan_sizes(n: int, t_block: int) -> Sizes:
    s = Sizes()
    rc = load().bload_plan_sizes(n, t_block, C.byref(s))
    if rc:
        raise BloadError(rc, "bload_plan_sizes")
    return s


@dataclass
class Plan:
    """A device plan: the raw buffer, its host scalars, and typed views of its tables (device tensors
    that alias the buffer)."""
    buf: "object"
    info: PlanInfo
    sizes: Sizes

    def _view(self, off: int, count: int, dtype):
        import torch
        esz = torch.empty((), dtype=dtype).element_size()
        return self.buf[off: off + count * esz].view(dtype)

    @property
    def n(self): return int(self.info.n)
    @property
    def t_block(self): return int(self.info.t_block)
    @property
    def n_blocks(self): return int(self.info.n_blocks)
    @property
    def sum_t(self): return int(self.info.sum_t)

    def tables(self) -> dict:
        import torch
        n, nb, s = self.n, self.n_blocks, self.sizes
        return dict(
            offsets=self._view(s.off_offsets, n + 1, torch.int64),
            seg_seq=self._view(s.off_seg_seq, n, torch.int32),
            seg_block=self._view(s.off_seg_block, n, torch.int32),
            seg_start=self._view(s.off_seg_start, n, torch.int32),
            seg_src=self._view(s.off_seg_src, n, torch.int64),
            block_seg_begin=self._view(s.off_block_seg_begin, nb + 1, torch.int32),
            block_fill=self._view(s.off_block_fill, nb, torch.int32),
            seq_block=self._view(s.off_seq_block, n, torch.int32),
            seq_start=self._view(s.off_seq_start, n, torch.int32),
        )


def bload_plan(lengths, t_block: int, seed: int, policy: int = 0, stream=None, work=None, plan_buf=None,
               check: bool = True) -> Plan:
    """lengths: CUDA int32 tensor [n].  Returns a Plan whose tables live in device memory."""
    import torch
    if not lengths.is_cuda or lengths.dtype != torch.int32 or not lengths.is_contiguous():
        raise TypeError("lengths must be a contiguous CUDA int32 tensor")
    n = lengths.numel()
    sizes = bload_plan_sizes(n, t_block)
    dev = lengths.device
    if plan_buf is None:
        plan_buf = torch.empty(sizes.plan_bytes, dtype=torch.uint8, device=dev)
    if work is None:
        work = torch.empty(sizes.work_bytes, dtype=torch.uint8, device=dev)
    info = PlanInfo()
    rc = load().bload_plan(lengths.data_ptr(), n, t_block, seed, policy, plan_buf.data_ptr(), plan_buf.numel(),
                           work.data_ptr(), work.numel(), _stream(stream), C.byref(info))
    if rc and check:
        err = BloadError(rc, "bload_plan")
        err.info = info
        raise err
    return Plan(plan_buf, info, sizes)


def bload_epoch(lengths, t_block: int, seed: int, block_capacity: int, store=None, frame_bytes: int = 0, dense=None,
                seq_id=None, pos=None, reset=None, valid=None, pad_byte: int = 0, dense_out=None,
                out_frame_bytes: int = 0, ragged_out=None, stream=None, side_stream=None, work=None, plan_buf=None,
                check: bool = True, chunks: int = 0) -> Plan:
    """Plan, metadata, pack and unpack of a whole epoch in one call; the copies of finished blocks run on
    `side_stream` while the plan is still being built on `stream`.  Same results as bload_plan + bload_pack +
    bload_unpack over blocks [0, block_capacity).  All outputs are complete when the call returns."""
    import torch
    if not lengths.is_cuda or lengths.dtype != torch.int32 or not lengths.is_contiguous():
        raise TypeError("lengths must be a contiguous CUDA int32 tensor")
    n = lengths.numel()
    sizes = bload_plan_sizes(n, t_block)
    if plan_buf is None:
        plan_buf = torch.empty(sizes.plan_bytes, dtype=torch.uint8, device=lengths.device)
    if work is None:
        work = torch.empty(sizes.work_bytes, dtype=torch.uint8, device=lengths.device)
    io = EpochIO(_ptr(store), frame_bytes, _ptr(dense), _ptr(seq_id), _ptr(pos), _ptr(reset), _ptr(valid),
                 _ptr(dense_out), out_frame_bytes, _ptr(ragged_out), block_capacity, pad_byte, chunks)
    info = PlanInfo()
    side = None if side_stream is None else (side_stream.cuda_stream or None)
    rc = load().bload_epoch(lengths.data_ptr(), n, t_block, seed, plan_buf.data_ptr(), plan_buf.numel(),
                            work.data_ptr(), work.numel(), C.byref(io), _stream(stream), side, C.byref(info))
    if rc and check:
        err = BloadError(rc, "bload_epoch")
        err.info = info
        raise err
    return Plan(plan_buf, info, sizes)


def bload_epoch_stage_times() -> list[float]:
    out = (C.c_float * 5)()
    rc = load().bload_epoch_stage_times(C.byref(out))
    if rc:
        raise BloadError(rc, "bload_epoch_stage_times")
    return [float(x) for x in out]


def bload_plan_async(lengths, t_block: int, seed: int, policy: int = 0, stream=None, work=None, plan_buf=None):
    """Enqueue a plan without waiting for it.  Returns (plan_buf, work, sizes); keep all three alive and
    call bload_plan_finish(plan_buf, sizes, stream) to obtain the Plan."""
    import torch
    if not lengths.is_cuda or lengths.dtype != torch.int32 or not lengths.is_contiguous():
        raise TypeError("lengths must be a contiguous CUDA int32 tensor")
    n = lengths.numel()
    sizes = bload_plan_sizes(n, t_block)
    if plan_buf is None:
        plan_buf = torch.empty(sizes.plan_bytes, dtype=torch.uint8, device=lengths.device)
    if work is None:
        work = torch.empty(sizes.work_bytes, dtype=torch.uint8, device=lengths.device)
    rc = load().bload_plan_async(lengths.data_ptr(), n, t_block, seed, policy, plan_buf.data_ptr(), plan_buf.numel(),
                                 work.data_ptr(), work.numel(), _stream(stream))
    if rc:
        raise BloadError(rc, "bload_plan_async")
    return plan_buf, work, sizes


def bload_plan_finish(plan_buf, sizes: Sizes, stream=None, check: bool = True) -> Plan:
    info = PlanInfo()
    rc = load().bload_plan_finish(plan_buf.data_ptr(), _stream(stream), C.byref(info))
    if rc and check:
        err = BloadError(rc, "bload_plan_finish")
        err.info = info
        raise err
    return Plan(plan_buf, info, sizes)


def bload_pack(plan: Plan, store, frame_bytes: int, block_begin: int, block_count: int, dense=None, seq_id=None,
               pos=None, reset=None, valid=None, pad_byte: int = 0, stream=None, repeat_last: bool = False) -> None:
    """store: CUDA tensor holding the flat ragged frames; dense/seq_id/pos/reset/valid: CUDA outputs or None.
    repeat_last: padding slots repeat the block's last frame (bload_pack_repeat_last) instead of pad_byte."""
    fn = load().bload_pack_repeat_last if repeat_last else load().bload_pack
    rc = fn(plan.buf.data_ptr(), C.byref(plan.info), _ptr(store), frame_bytes, block_begin,
                           block_count, _ptr(dense), _ptr(seq_id), _ptr(pos), _ptr(reset), _ptr(valid), pad_byte,
                           _stream(stream))
    if rc:
        raise BloadError(rc, "bload_pack")


def bload_unpack(plan: Plan, dense_out, out_frame_bytes: int, block_begin: int, block_count: int, ragged_out,
                 stream=None) -> None:
    rc = load().bload_unpack(plan.buf.data_ptr(), C.byref(plan.info), _ptr(dense_out), out_frame_bytes, block_begin,
                             block_count, _ptr(ragged_out), _stream(stream))
    if rc:
        raise BloadError(rc, "bload_unpack")


def bload_var_offsets(lengths, frame_bytes, stream=None):
    """Byte offsets of a store whose sequence i holds lengths[i] frames of frame_bytes[i] bytes (CUDA int32 tensors).
    Returns (byte_offsets int64 CUDA tensor [n+3], VarInfo); the first n+1 entries are the offsets."""
    import torch
    n = lengths.numel()
    out = torch.empty(n + 3, dtype=torch.int64, device=lengths.device)
    info = VarInfo()
    rc = load().bload_var_offsets(lengths.data_ptr(), frame_bytes.data_ptr(), n, out.data_ptr(), _stream(stream),
                                  C.byref(info))
    if rc:
        err = BloadError(rc, "bload_var_offsets")
        err.info = info
        raise err
    return out, info


def bload_pack_var(plan: Plan, store, frame_bytes, byte_offsets, slot_bytes: int, block_begin: int, block_count: int,
                   dense, pad_byte: int = 0, stream=None) -> None:
    rc = load().bload_pack_var(plan.buf.data_ptr(), C.byref(plan.info), _ptr(store), _ptr(frame_bytes),
                               _ptr(byte_offsets), slot_bytes, block_begin, block_count, _ptr(dense), pad_byte,
                               _stream(stream))
    if rc:
        raise BloadError(rc, "bload_pack_var")


def bload_unpack_var(plan: Plan, dense_out, frame_bytes, byte_offsets, slot_bytes: int, block_begin: int,
                     block_count: int, ragged_out, stream=None) -> None:
    rc = load().bload_unpack_var(plan.buf.data_ptr(), C.byref(plan.info), _ptr(dense_out), _ptr(frame_bytes),
                                 _ptr(byte_offsets), slot_bytes, block_begin, block_count, _ptr(ragged_out),
                                 _stream(stream))
    if rc:
        raise BloadError(rc, "bload_unpack_var")


def bload_var_offsets2d(lengths, rows, row_bytes, stream=None):
    """Byte offsets of a store whose sequence i holds lengths[i] images of rows[i] x row_bytes[i] bytes.
    Returns (byte_offsets int64 CUDA tensor [n+4], VarInfo)."""
    import torch
    n = lengths.numel()
    out = torch.empty(n + 4, dtype=torch.int64, device=lengths.device)
    info = VarInfo()
    rc = load().bload_var_offsets2d(lengths.data_ptr(), rows.data_ptr(), row_bytes.data_ptr(), n, out.data_ptr(),
                                    _stream(stream), C.byref(info))
    if rc:
        err = BloadError(rc, "bload_var_offsets2d")
        err.info = info
        raise err
    return out, info


def bload_pack_var2d(plan: Plan, store, rows, row_bytes, byte_offsets, rows_max: int, row_stride: int,
                     block_begin: int, block_count: int, dense, pad_byte: int = 0, stream=None) -> None:
    rc = load().bload_pack_var2d(plan.buf.data_ptr(), C.byref(plan.info), _ptr(store), _ptr(rows), _ptr(row_bytes),
                                 _ptr(byte_offsets), rows_max, row_stride, block_begin, block_count, _ptr(dense),
                                 pad_byte, _stream(stream))
    if rc:
        raise BloadError(rc, "bload_pack_var2d")


def bload_unpack_var2d(plan: Plan, dense_out, rows, row_bytes, byte_offsets, rows_max: int, row_stride: int,
                       block_begin: int, block_count: int, ragged_out, stream=None) -> None:
    rc = load().bload_unpack_var2d(plan.buf.data_ptr(), C.byref(plan.info), _ptr(dense_out), _ptr(rows),
                                   _ptr(row_bytes), _ptr(byte_offsets), rows_max, row_stride, block_begin, block_count,
                                   _ptr(ragged_out), _stream(stream))
    if rc:
        raise BloadError(rc, "bload_unpack_var2d")


def bload_carry_prev(plan: Plan, dense, frame_bytes: int, block_begin: int, block_count: int, prev,
                     fill_byte: int = 0, stream=None) -> None:
    """prev[q, s] = dense[q, s-1] where a sequence continues at slot s, fill_byte elsewhere (CUDA tensors)."""
    rc = load().bload_carry_prev(plan.buf.data_ptr(), C.byref(plan.info), _ptr(dense), frame_bytes, block_begin,
                                 block_count, _ptr(prev), fill_byte, _stream(stream))
    if rc:
        raise BloadError(rc, "bload_carry_prev")


def bload_reset_state(plan: Plan, block_begin: int, block_count: int, slot: int, state, state_bytes: int,
                      init=None, stream=None) -> None:
    """Re-initialise, in place, the rows of `state` whose block does not continue a sequence at `slot`."""
    rc = load().bload_reset_state(plan.buf.data_ptr(), C.byref(plan.info), block_begin, block_count, slot,
                                  _ptr(state), state_bytes, _ptr(init), _stream(stream))
    if rc:
        raise BloadError(rc, "bload_reset_state")


def bload_valid_sum(plan: Plan, values, block_begin: int, block_count: int, block_sum, total=None,
                    stream=None) -> None:
    """block_sum[q] (float64 CUDA tensor) = sum of the float32 values on the frames of block q; total = [sum, frames]."""
    rc = load().bload_valid_sum(plan.buf.data_ptr(), C.byref(plan.info), _ptr(values), block_begin, block_count,
                                _ptr(block_sum), _ptr(total), _stream(stream))
    if rc:
        raise BloadError(rc, "bload_valid_sum")


def bload_stats(info: PlanInfo) -> dict:
    s = Stats()
    rc = load().bload_stats(C.byref(info), C.byref(s))
    if rc:
        raise BloadError(rc, "bload_stats")
    return {k: getattr(s, k) for k, _ in Stats._fields_}


def bload_set_plan_timing(enable: bool) -> None:
    load().bload_set_plan_timing(1 if enable else 0)


def bload_plan_stage_times() -> list[float]:
    out = (C.c_float * 4)()
    rc = load().bload_plan_stage_times(C.byref(out))
    if rc:
        raise BloadError(rc, "bload_plan_stage_times")
    return [float(x) for x in out]


def bload_kernel_launches() -> int:
    return int(load().bload_kernel_launches())


def bload_debug_status(clear: bool = False):
    """[refused accesses, kernel number of the first, 0 read / 1 write, address] of the bounds-checking build
    (BLOAD_LIBRARY=.../libbload_debug.so); None from the ordinary build."""
    out = (C.c_uint64 * 4)()
    rc = load().bload_debug_status(C.byref(out), 1 if clear else 0)
    if rc == ERR_UNSUPPORTED:
        return None
    if rc:
        raise BloadError(rc, "bload_debug_status")
    return [int(x) for x in out]


KEEP_TAIL, DROP_TAIL = 0, 1


def bload_plan_chunks(lengths, t_chunk: int, tail: int = KEEP_TAIL, stream=None, check: bool = True):
    """The chunking strategy of the paper's comparison ("sampling"): every chunk of t_chunk frames of every sequence is a
    sample and a block.  Returns (Plan over the chunks, ChunkInfo, chunk_seq, chunk_first); the two int32 CUDA tensors
    name, per chunk, the sequence it was cut from and its first frame there.  Two calls into the library: the count
    (the plan cannot be sized before it), then the plan."""
    import torch
    if not lengths.is_cuda or lengths.dtype != torch.int32 or not lengths.is_contiguous():
        raise TypeError("lengths must be a contiguous CUDA int32 tensor")
    n = lengths.numel()
    L = load()
    work = torch.empty(max(int(L.bload_chunk_work_bytes(n)), 256), dtype=torch.uint8, device=lengths.device)
    ci = ChunkInfo()
    rc = L.bload_chunk_count(lengths.data_ptr(), n, t_chunk, tail, work.data_ptr(), work.numel(), _stream(stream), C.byref(ci))
    if rc:
        err = BloadError(rc, "bload_chunk_count")
        err.info = ci
        if check:
            raise err
        return None, ci, None, None
    m = int(ci.n_chunks)
    if m < 1:
        if check:
            raise BloadError(ERR_ARG, "bload_plan_chunks (no chunk is kept)")
        return None, ci, None, None
    sizes = bload_plan_sizes(m, t_chunk)
    plan_buf = torch.empty(sizes.plan_bytes, dtype=torch.uint8, device=lengths.device)
    chunk_seq = torch.empty(m, dtype=torch.int32, device=lengths.device)
    chunk_first = torch.empty(m, dtype=torch.int32, device=lengths.device)
    info = PlanInfo()
    rc = L.bload_plan_chunks(lengths.data_ptr(), n, t_chunk, tail, m, plan_buf.data_ptr(), plan_buf.numel(), work.data_ptr(),
                             work.numel(), chunk_seq.data_ptr(), chunk_first.data_ptr(), _stream(stream), C.byref(info))
    if rc and check:
        err = BloadError(rc, "bload_plan_chunks")
        err.info = info
        raise err
    return Plan(plan_buf, info, sizes), ci, chunk_seq, chunk_first


COPY_CALLS = {"pack": 0, "unpack": 1, "carry_prev": 2, "pack_var": 3, "unpack_var": 4}


def bload_last_copy_kernel(which: str) -> str:
    """Name of the copy kernel the last bload_pack / unpack / carry_prev / pack_var / unpack_var call of this thread chose."""
    return load().bload_last_copy_kernel(COPY_CALLS[which]).decode()


STATIC_MAX_N = 65536


def bload_plan_static(lengths, t_block: int, seed: int, policy: int = 0, stream=None, plan_buf=None,
                      check: bool = True) -> Plan:
    """bload_plan without a caller-provided scratch buffer, for callers that cannot allocate device
    memory (for example a loader thread beside a training job whose allocator owns the device).
    The library's built-in scratch array is used instead, which caps n at STATIC_MAX_N; calls that
    overlap on the GPU race on that array.  policy: 0 or 1 (best fit decreasing, 2, does not fit the
    array and raises ERR_UNSUPPORTED).  Pass a pre-made `plan_buf` to avoid every allocation; without
    one this wrapper (not the library) allocates the plan buffer with torch."""
    import torch
    if not lengths.is_cuda or lengths.dtype != torch.int32 or not lengths.is_contiguous():
        raise TypeError("lengths must be a contiguous CUDA int32 tensor")
    fn = load().bload_plan_static
    n = lengths.numel()
    sizes = bload_plan_sizes(n, t_block)
    if plan_buf is None:
        plan_buf = torch.empty(sizes.plan_bytes, dtype=torch.uint8, device=lengths.device)
    info = PlanInfo()
    rc = fn(lengths.data_ptr(), n, t_block, seed, policy, plan_buf.data_ptr(), plan_buf.numel(), _stream(stream),
            C.byref(info))
    if rc and check:
        err = BloadError(rc, "bload_plan_static")
        err.info = info
        raise err
    return Plan(plan_buf, info, sizes)


def bload_rank_range(n_blocks: int, world_size: int, rank: int, batch_blocks: int = 1) -> tuple[int, int]:
    """(first block, number of blocks) of one data-parallel rank; the same count on every rank, rounded up to whole
    batches (blocks beyond n_blocks are packed as padding)."""
    b, c = C.c_int64(), C.c_int64()
    rc = load().bload_rank_range(n_blocks, world_size, rank, batch_blocks, C.byref(b), C.byref(c))
    if rc:
        raise BloadError(rc, "bload_rank_range")
    return int(b.value), int(c.value)


# ---- layers on packed batches: everything below takes the per-slot positions that bload_pack writes ----------------
# The calls write into the tensors they are given and are not recorded by autograd; each has a gradient call of its own.

F32, F16, BF16 = 0, 1, 2
RECURRENCE_RUN = 64


class HeadsTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("block_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64)]


class AttentionArgs(C.Structure):
    _fields_ = [("block_count", C.c_int64), ("t_block", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("dtype", C.c_int32), ("causal", C.c_int32), ("window", C.c_int32),
                ("scale", C.c_float), ("softcap", C.c_float), ("d_pos", C.c_void_p), ("d_slopes", C.c_void_p),
                ("q", HeadsTensor), ("k", HeadsTensor), ("v", HeadsTensor), ("out", HeadsTensor), ("d_lse", C.c_void_p),
                ("dout", HeadsTensor), ("dq", HeadsTensor), ("dk", HeadsTensor), ("dv", HeadsTensor),
                ("d_delta", C.c_void_p)]


class ChannelsTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("block_stride", C.c_int64), ("slot_stride", C.c_int64)]


class RecurrenceArgs(C.Structure):
    _fields_ = [("block_count", C.c_int64), ("channels", C.c_int64), ("t_block", C.c_int32), ("dtype", C.c_int32),
                ("d_pos", C.c_void_p), ("gate", ChannelsTensor), ("x", ChannelsTensor), ("h", ChannelsTensor),
                ("d_carry", C.c_void_p), ("d_work", C.c_void_p), ("work_bytes", C.c_size_t), ("dh", ChannelsTensor),
                ("dgate", ChannelsTensor), ("dx", ChannelsTensor)]


class NormArgs(C.Structure):
    _fields_ = [("block_count", C.c_int64), ("channels", C.c_int64), ("t_block", C.c_int32), ("dtype", C.c_int32),
                ("eps", C.c_float), ("d_pos", C.c_void_p), ("d_weight", C.c_void_p), ("d_bias", C.c_void_p),
                ("d_stats", C.c_void_p), ("x", ChannelsTensor), ("y", ChannelsTensor), ("dy", ChannelsTensor),
                ("dx", ChannelsTensor), ("d_dweight", C.c_void_p), ("d_dbias", C.c_void_p), ("d_work", C.c_void_p),
                ("work_bytes", C.c_size_t)]


class ConvArgs(C.Structure):
    _fields_ = [("block_count", C.c_int64), ("channels", C.c_int64), ("t_block", C.c_int32), ("dtype", C.c_int32),
                ("taps", C.c_int32), ("silu", C.c_int32), ("d_pos", C.c_void_p), ("d_weight", C.c_void_p),
                ("d_bias", C.c_void_p), ("x", ChannelsTensor), ("y", ChannelsTensor), ("d_seq_id", C.c_void_p),
                ("n_seq", C.c_int64), ("d_tails", C.c_void_p), ("dy", ChannelsTensor), ("dx", ChannelsTensor),
                ("d_dweight", C.c_void_p), ("d_dbias", C.c_void_p), ("d_work", C.c_void_p), ("work_bytes", C.c_size_t)]


class ScanArgs(C.Structure):
    _fields_ = [("block_count", C.c_int64), ("channels", C.c_int64), ("t_block", C.c_int32), ("dtype", C.c_int32),
                ("states", C.c_int32), ("softplus", C.c_int32), ("d_pos", C.c_void_p), ("d_a", C.c_void_p), ("d_d", C.c_void_p),
                ("d_dt_bias", C.c_void_p)] + [(n, ChannelsTensor) for n in ("x", "dt", "b", "c", "z", "y")] + \
               [("d_carry", C.c_void_p), ("d_work", C.c_void_p), ("work_bytes", C.c_size_t), ("d_seq_id", C.c_void_p),
                ("n_seq", C.c_int64), ("d_last", C.c_void_p)] + \
               [(n, ChannelsTensor) for n in ("dy", "dx", "ddt", "db", "dc", "dz")] + \
               [("d_da", C.c_void_p), ("d_dd", C.c_void_p), ("d_ddt_bias", C.c_void_p)]


class ScanStepArgs(C.Structure):
    _fields_ = [("rows", C.c_int64), ("channels", C.c_int64), ("dtype", C.c_int32), ("states", C.c_int32), ("softplus", C.c_int32),
                ("d_pos", C.c_void_p), ("d_a", C.c_void_p), ("d_d", C.c_void_p), ("d_dt_bias", C.c_void_p),
                ("state", C.c_void_p), ("next", C.c_void_p)] + [(n, ChannelsTensor) for n in ("x", "dt", "b", "c", "z", "y")]


# The argument blocks of a call, packed in one step: these calls are made per layer and step, and filling a ctypes structure
# field by field takes longer than the kernels of a small batch.  (The layouts are those of the structures above.)
_HEADS = struct.Struct("@4q")
_ATTENTION = struct.Struct("@q7i2fi2q16qq")
_ATTENTION_GRAD = struct.Struct("@q7i2fi2q16qq16qq")
_RECURRENCE = struct.Struct("@2q2iq9q2qQ9q")
_CHANNELS = struct.Struct("@3q")
_NORM = struct.Struct("@2q2if4q6q6q3qQ")
_CONV = struct.Struct("@2q4i3q6q3q6q3qQ")
_SCAN = struct.Struct("@2q4i4q18q2qQ3q18q3q")
_SCAN_STEP = struct.Struct("@2q3i6q18q")


def _torch():
    """({dtype: code}, int32, float32, raw stream of a device, current device, uint8) of torch, looked up once."""
    global _torch_parts
    if _torch_parts is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _torch_parts = ({torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}, torch.int32, torch.float32,
                        raw or (lambda index: torch.cuda.current_stream(index).cuda_stream), torch.cuda.current_device, torch.uint8)
    return _torch_parts


_torch_parts = None


def _begin(where: str, pos, x, dims: int, stream):
    """Checks of the positions and the leading tensor; ((blocks, t_block), element type code, stream)."""
    codes, int32, _, raw_stream, current_device, _ = _torch()
    index = pos.get_device()
    if pos.dtype is not int32 or pos.dim() != 2 or index < 0 or not pos.is_contiguous():
        raise TypeError("%s: pos must be a contiguous CUDA int32 tensor [blocks, t_block], as bload_pack writes it" % where)
    if index != current_device():
        raise ValueError("%s: pos is on %s, the current device is cuda:%d" % (where, pos.device, current_device()))
    if x.dim() != dims or x.get_device() != index:
        raise ValueError("%s: tensors are [blocks, t_block, %s] on the device of pos" % (where, "heads, head_dim" if dims == 4 else "channels"))
    code = codes.get(x.dtype)
    if code is None:
        raise TypeError("%s: float32, float16 or bfloat16 tensors, not %s" % (where, x.dtype))
    return pos.shape, code, raw_stream(index) if stream is None else stream.cuda_stream


def _strided(where: str, name: str, t, shape, like):
    """(address, strides but the last) of a strided tensor argument; the last dimension has to be contiguous."""
    if t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise TypeError("%s: %s is %s on %s, expected %s on %s" % (where, name, t.dtype, t.device, like.dtype, like.device))
    if t.shape != shape:
        raise ValueError("%s: %s has shape %s, expected %s" % (where, name, tuple(t.shape), tuple(shape)))
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise ValueError("%s: the last dimension of %s must be contiguous" % (where, name))
    return (t.data_ptr(), *st[:-1])


def _flat32(where: str, name: str, t, count: int, like) -> int:
    """Address of a contiguous float32 argument, 0 for None."""
    if t is None:
        return 0
    if t.dtype is not _torch()[2] or t.get_device() != like.get_device() or not t.is_contiguous() or t.numel() != count:
        raise TypeError("%s: %s must be a contiguous float32 tensor of %d elements on %s" % (where, name, count, like.device))
    return t.data_ptr()


def _rotary(fn, where, pos, x, y, inv_freq, interleaved, factor, stream) -> None:
    (b, t), code, stream = _begin(where, pos, x, 4, stream)
    h, d = x.shape[2:]
    shape = (b, t, h, d)
    n = inv_freq.numel()
    rc = fn(pos.data_ptr(), b, t, h, d, code, _HEADS.pack(*_strided(where, "input", x, shape, x)),
            _HEADS.pack(*_strided(where, "output", y, shape, x)), _flat32(where, "inv_freq", inv_freq, n, x), 2 * n,
            1 if interleaved else 0, factor, stream)
    if rc:
        raise BloadError(rc, where)


def bload_rotary(pos, x, y, inv_freq, interleaved: bool = False, factor: float = 1.0, stream=None) -> None:
    """y = rotary positions applied to x [blocks, t_block, heads, head_dim] (strided; y may be x).  pos: int32 [blocks,
    t_block] from bload_pack; inv_freq: float32 [rot_dim / 2], the elements from rot_dim on are copied."""
    _rotary(load().bload_rotary, "bload_rotary", pos, x, y, inv_freq, interleaved, factor, stream)


def bload_rotary_grad(pos, dy, dx, inv_freq, interleaved: bool = False, factor: float = 1.0, stream=None) -> None:
    """dx = gradient of bload_rotary's input, from the gradient dy of its output (dx may be dy)."""
    _rotary(load().bload_rotary_grad, "bload_rotary_grad", pos, dy, dx, inv_freq, interleaved, factor, stream)


def _attention(where, pos, q, k, v, out, lse, scale, softcap, slopes, causal, window, stream):
    """(packed fields up to d_lse, stream)"""
    (b, t), code, stream = _begin(where, pos, q, 4, stream)
    h, d = q.shape[2:]
    if k.dim() != 4:
        raise ValueError("%s: k and v are [blocks, t_block, kv_heads, head_dim]" % where)
    hk = k.shape[2]
    qs, ks = (b, t, h, d), (b, t, hk, d)
    return (b, t, h, hk, d, code, 1 if causal else 0, window, d ** -0.5 if scale is None else scale, softcap, 0,
            pos.data_ptr(), _flat32(where, "slopes", slopes, h, q), *_strided(where, "q", q, qs, q),
            *_strided(where, "k", k, ks, q), *_strided(where, "v", v, ks, q), *_strided(where, "out", out, qs, q),
            _flat32(where, "lse", lse, b * h * t, q)), stream


def bload_attention(pos, q, k, v, out, lse=None, scale: float | None = None, softcap: float = 0.0, slopes=None,
                    causal: bool = True, window: int = 0, stream=None) -> None:
    """Attention inside the sequences of packed blocks.  q, out: [blocks, t_block, heads, head_dim], k, v: [.., kv_heads, ..]
    (float16 or bfloat16, strided); pos: int32 [blocks, t_block] from bload_pack; lse: float32 [blocks, heads, t_block] or
    None (needed for the gradient).  scale defaults to head_dim ** -0.5; softcap > 0 caps scores by a tanh; slopes: float32
    [heads], subtracts slope * |i - j|; window > 0 keeps |i - j| < window."""
    fields, stream = _attention("bload_attention", pos, q, k, v, out, lse, scale, softcap, slopes, causal, window, stream)
    rc = load().bload_attention(_ATTENTION.pack(*fields), stream)
    if rc:
        raise BloadError(rc, "bload_attention")


def bload_attention_grad(pos, q, k, v, out, lse, dout, dq, dk, dv, delta, scale: float | None = None, softcap: float = 0.0,
                         slopes=None, causal: bool = True, window: int = 0, stream=None) -> None:
    """dq, dk, dv of bload_attention from dout, with out and lse of the forward call.  delta: float32 [blocks, heads,
    t_block], written (the row sums of dout * out, without the rounding of out)."""
    where = "bload_attention_grad"
    fields, stream = _attention(where, pos, q, k, v, out, lse, scale, softcap, slopes, causal, window, stream)
    rc = load().bload_attention_grad(_ATTENTION_GRAD.pack(
        *fields, *_strided(where, "dout", dout, q.shape, q), *_strided(where, "dq", dq, q.shape, q),
        *_strided(where, "dk", dk, k.shape, q), *_strided(where, "dv", dv, k.shape, q),
        _flat32(where, "delta", delta, q.shape[0] * q.shape[1] * q.shape[2], q)), stream)
    if rc:
        raise BloadError(rc, where)


def bload_recurrence_buffers(pos, x):
    """(carry, work) for bload_recurrence and its gradient on x [blocks, t_block, channels]: the float32 states that the
    forward call keeps for the gradient, [blocks, ceil(t_block / 64), channels], and scratch (None when none is needed).
    Calls that may overlap on the GPU need a scratch each."""
    b, t = pos.shape
    c = x.shape[-1]
    n = load().bload_recurrence_work_bytes(b, t, c)
    new = x.new_empty
    return (new((b, -(-t // RECURRENCE_RUN), c), dtype=_torch()[2]),
            new(n, dtype=_torch()[5]) if n else None)


def _recurrence(where, pos, gate, x, carry, work, stream):
    """(packed fields up to x, of d_carry to work_bytes, stream)"""
    (b, t), code, stream = _begin(where, pos, x, 3, stream)
    c = x.shape[2]
    head = (b, c, t, code, pos.data_ptr(), *_strided(where, "gate", gate, x.shape, x), *_strided(where, "x", x, (b, t, c), x))
    at = _flat32(where, "carry", carry, b * -(-t // RECURRENCE_RUN) * c, x)
    if work is None:
        return head, (at, 0, 0), stream
    if work.device != x.device or not work.is_contiguous():
        raise TypeError("%s: work must be a contiguous tensor on %s" % (where, x.device))
    return head, (at, work.data_ptr(), work.numel() * work.element_size()), stream


def bload_recurrence(pos, gate, x, h, carry=None, work=None, stream=None) -> None:
    """h_s = f_s h_{s-1} + (1 - f_s) x_s with f = sigmoid(gate), restarted at every sequence start.  gate, x, h: [blocks,
    t_block, channels] (float32, float16 or bfloat16, strided); carry, work from bload_recurrence_buffers (carry None:
    no gradient will be asked for)."""
    where = "bload_recurrence"
    head, kept, stream = _recurrence(where, pos, gate, x, carry, work, stream)
    rc = load().bload_recurrence(_RECURRENCE.pack(*head, *_strided(where, "h", h, x.shape, x), *kept, 0, 0, 0, 0, 0, 0, 0, 0, 0), stream)
    if rc:
        raise BloadError(rc, where)


def bload_recurrence_grad(pos, gate, x, carry, dh, dgate, dx, work=None, stream=None) -> None:
    """dgate and dx of bload_recurrence from dh, the gradient with respect to every h; carry is the forward call's."""
    where = "bload_recurrence_grad"
    head, kept, stream = _recurrence(where, pos, gate, x, carry, work, stream)
    rc = load().bload_recurrence_grad(_RECURRENCE.pack(
        *head, 0, 0, 0, *kept, *_strided(where, "dh", dh, x.shape, x), *_strided(where, "dgate", dgate, x.shape, x),
        *_strided(where, "dx", dx, x.shape, x)), stream)
    if rc:
        raise BloadError(rc, where)


def _axes(fn, where, pos, coords, axis, x, y, inv_freq, interleaved, factor, stream) -> None:
    (b, t), code, stream = _begin(where, pos, x, 4, stream)
    h, d = x.shape[2:]
    shape, n = (b, t, h, d), inv_freq.numel()
    for name, given, want in (("coords", coords, coords.dim() == 3 and coords.shape[1:] == pos.shape), ("axis", axis, axis.numel() == n)):
        if given.dtype is not pos.dtype or given.get_device() != pos.get_device() or not given.is_contiguous():
            raise TypeError("%s: %s must be a contiguous int32 tensor on %s" % (where, name, pos.device))
        if not want:
            raise ValueError("%s: coords is [axes, blocks, t_block], axis has an axis for each of inv_freq's pairs" % where)
    rc = fn(pos.data_ptr(), coords.data_ptr(), coords.shape[0], axis.data_ptr(), b, t, h, d, code,
            _HEADS.pack(*_strided(where, "input", x, shape, x)), _HEADS.pack(*_strided(where, "output", y, shape, x)),
            _flat32(where, "inv_freq", inv_freq, n, x), 2 * n, 1 if interleaved else 0, factor, stream)
    if rc:
        raise BloadError(rc, where)


def bload_rotary_axes(pos, coords, axis, x, y, inv_freq, interleaved: bool = False, factor: float = 1.0, stream=None) -> None:
    """Rotary positions with several axes (video: time, height, width): pair i of every head of x [blocks, t_block, heads,
    head_dim] turns by coords[axis[i]] * inv_freq[i] into y (which may be x).  coords: int32 [axes, blocks, t_block], at most
    4 axes; axis: int32, one per element of inv_freq; pos: int32 [blocks, t_block] from bload_pack, whose padding is copied."""
    _axes(load().bload_rotary_axes, "bload_rotary_axes", pos, coords, axis, x, y, inv_freq, interleaved, factor, stream)


def bload_rotary_axes_grad(pos, coords, axis, dy, dx, inv_freq, interleaved: bool = False, factor: float = 1.0, stream=None) -> None:
    """dx = gradient of bload_rotary_axes's input, from the gradient dy of its output (dx may be dy)."""
    _axes(load().bload_rotary_axes_grad, "bload_rotary_axes_grad", pos, coords, axis, dy, dx, inv_freq, interleaved, factor, stream)


_NONE3, _NONE6, _NONE18 = (0,) * 3, (0,) * 6, (0,) * 18


def _work(where: str, work, like):
    """(address, bytes) of a scratch argument"""
    if work is None:
        return 0, 0
    if work.get_device() != like.get_device() or not work.is_contiguous():
        raise TypeError("%s: work must be a contiguous tensor on %s" % (where, like.device))
    return work.data_ptr(), work.numel() * work.element_size()


def _sequences(where: str, pos, seq_id, out, name: str, shape, dtype):
    """(address of the sequence numbers, how many, address of the output) of a call that writes something per sequence"""
    if out is None:
        return 0, 0, 0
    if seq_id is None or seq_id.dtype is not pos.dtype or seq_id.shape != pos.shape or seq_id.get_device() != pos.get_device() or not seq_id.is_contiguous():
        raise TypeError("%s: %s needs seq_id, a contiguous int32 tensor like pos, as bload_pack writes it" % (where, name))
    if out.dtype is not dtype or out.get_device() != pos.get_device() or not out.is_contiguous() or out.dim() != 3 or out.shape[1:] != shape:
        raise TypeError("%s: %s must be a contiguous %s tensor [sequences, %d, %d] on %s" % (where, name, dtype, *shape, pos.device))
    return seq_id.data_ptr(), out.shape[0], out.data_ptr()


def bload_norm_buffers(pos, x):
    """(stats, work) for bload_norm and its gradient on x [blocks, t_block, channels]: float32 [blocks, t_block, 2], means and
    reciprocal deviations that the forward call keeps, and the gradient's scratch."""
    b, t = pos.shape
    n = load().bload_norm_work_bytes(b, t, x.shape[-1], _torch()[0].get(x.dtype, -1))
    return x.new_empty((b, t, 2), dtype=_torch()[2]), x.new_empty(n, dtype=_torch()[5]) if n else None


def _norm(where, pos, x, weight, bias, stats, eps, stream):
    """(packed fields up to x, stream)"""
    (b, t), code, stream = _begin(where, pos, x, 3, stream)
    c = x.shape[2]
    return (b, c, t, code, eps, pos.data_ptr(), _flat32(where, "weight", weight, c, x), _flat32(where, "bias", bias, c, x),
            _flat32(where, "stats", stats, b * t * 2, x), *_strided(where, "x", x, (b, t, c), x)), stream


def bload_norm(pos, x, y, weight=None, bias=None, stats=None, eps: float = 1e-5, stream=None) -> None:
    """y = layer norm of x over its channels, times weight plus bias (float32 [channels] or None); padding gives 0.  x, y: [blocks,
    t_block, channels] (float32, float16 or bfloat16, strided); pos: int32 [blocks, t_block] from bload_pack; stats from
    bload_norm_buffers (None: no gradient will be asked for)."""
    where = "bload_norm"
    fields, stream = _norm(where, pos, x, weight, bias, stats, eps, stream)
    rc = load().bload_norm(_NORM.pack(*fields, *_strided(where, "y", y, x.shape, x), *_NONE6, 0, 0, 0, 0), stream)
    if rc:
        raise BloadError(rc, where)


def bload_norm_grad(pos, x, stats, dy, dx, weight=None, dweight=None, dbias=None, work=None, stream=None) -> None:
    """dx of bload_norm from dy, with the forward call's stats, and the sums over all frames dweight and dbias (float32 [channels];
    None: not wanted, and neither is work then)."""
    where = "bload_norm_grad"
    fields, stream = _norm(where, pos, x, weight, None, stats, 0.0, stream)
    c = x.shape[2]
    rc = load().bload_norm_grad(_NORM.pack(
        *fields, *_NONE3, *_strided(where, "dy", dy, x.shape, x), *_strided(where, "dx", dx, x.shape, x),
        _flat32(where, "dweight", dweight, c, x), _flat32(where, "dbias", dbias, c, x), *_work(where, work, x)), stream)
    if rc:
        raise BloadError(rc, where)


def bload_conv_buffers(pos, x, weight):
    """Scratch of bload_conv_grad for x [blocks, t_block, channels] and weight [channels, taps]."""
    b, t = pos.shape
    n = load().bload_conv_work_bytes(b, t, x.shape[-1], weight.shape[-1], _torch()[0].get(x.dtype, -1))
    return x.new_empty(n, dtype=_torch()[5]) if n else None


def _conv(where, pos, x, weight, bias, silu, stream):
    """(packed fields up to x, stream)"""
    (b, t), code, stream = _begin(where, pos, x, 3, stream)
    c = x.shape[2]
    if weight.dim() != 2:
        raise ValueError("%s: weight is [channels, taps]" % where)
    taps = weight.shape[1]
    return (b, c, t, code, taps, 1 if silu else 0, pos.data_ptr(), _flat32(where, "weight", weight, c * taps, x),
            _flat32(where, "bias", bias, c, x), *_strided(where, "x", x, (b, t, c), x)), stream


def bload_conv(pos, x, y, weight, bias=None, silu: bool = True, seq_id=None, tails=None, stream=None) -> None:
    """y = short causal convolution of x [blocks, t_block, channels] per channel inside sequences, then u * sigmoid(u) if silu.
    weight: float32 [channels, taps], the last tap is the frame's own; bias: float32 [channels] or None; taps at most 8.  tails:
    [sequences, taps - 1, channels] like x or None: the last inputs of every sequence of the batch, numbered by seq_id (int32
    [blocks, t_block] from bload_pack), for bload_conv_step to go on from."""
    where = "bload_conv"
    fields, stream = _conv(where, pos, x, weight, bias, silu, stream)
    rc = load().bload_conv(_CONV.pack(*fields, *_strided(where, "y", y, x.shape, x),
                                      *_sequences(where, pos, seq_id, tails, "tails", (weight.shape[1] - 1, x.shape[2]), x.dtype),
                                      *_NONE6, 0, 0, 0, 0), stream)
    if rc:
        raise BloadError(rc, where)


def bload_conv_grad(pos, x, dy, dx, weight, dweight=None, bias=None, dbias=None, silu: bool = True, work=None, stream=None) -> None:
    """dx of bload_conv from dy, and the sums over all frames dweight [channels, taps] and dbias (float32; None: not wanted).  work
    from bload_conv_buffers."""
    where = "bload_conv_grad"
    fields, stream = _conv(where, pos, x, weight, bias, silu, stream)
    rc = load().bload_conv_grad(_CONV.pack(
        *fields, *_NONE3, 0, 0, 0, *_strided(where, "dy", dy, x.shape, x), *_strided(where, "dx", dx, x.shape, x),
        _flat32(where, "dweight", dweight, weight.numel(), x), _flat32(where, "dbias", dbias, x.shape[2], x), *_work(where, work, x)), stream)
    if rc:
        raise BloadError(rc, where)


def _rows(where: str, pos, x, stream):
    """Checks of a call for single frames; (rows, channels, element type code, stream)."""
    codes, int32, _, raw_stream, current_device, _ = _torch()
    index = pos.get_device()
    if pos.dtype is not int32 or pos.dim() != 1 or index < 0 or not pos.is_contiguous():
        raise TypeError("%s: pos must be a contiguous CUDA int32 tensor [rows]" % where)
    if index != current_device():
        raise ValueError("%s: pos is on %s, the current device is cuda:%d" % (where, pos.device, current_device()))
    if x.dim() != 2 or x.get_device() != index or x.shape[0] != pos.shape[0]:
        raise ValueError("%s: x is [rows, channels] on the device of pos" % where)
    code = codes.get(x.dtype)
    if code is None:
        raise TypeError("%s: float32, float16 or bfloat16 tensors, not %s" % (where, x.dtype))
    return (*x.shape, code, raw_stream(index) if stream is None else stream.cuda_stream)


def _state(where: str, name: str, t, shape, dtype, like) -> int:
    if t.dtype is not dtype or t.get_device() != like.get_device() or not t.is_contiguous() or t.shape != shape:
        raise TypeError("%s: %s must be a contiguous %s tensor %s on %s" % (where, name, dtype, tuple(shape), like.device))
    return t.data_ptr()


def bload_conv_step(pos, state, x, y, weight, bias=None, silu: bool = True, next_state=None, stream=None) -> None:
    """bload_conv for one new frame of each of several sequences: x, y [rows, channels]; state [rows, taps - 1, channels], the last
    inputs, moves on in place or into next_state.  pos: int32 [rows], positions of the new frames (0 starts a sequence, whatever
    the state holds; negative: no frame, y = 0 and the state stays)."""
    where = "bload_conv_step"
    n, c, code, stream = _rows(where, pos, x, stream)
    if weight.dim() != 2:
        raise ValueError("%s: weight is [channels, taps]" % where)
    taps = weight.shape[1]
    shape = (n, taps - 1, c)
    at = _state(where, "state", state, shape, x.dtype, x)
    to = at if next_state is None else _state(where, "next_state", next_state, shape, x.dtype, x)
    rc = load().bload_conv_step(n, c, code, taps, 1 if silu else 0, pos.data_ptr(), at, to,
                                _CHANNELS.pack(*_strided(where, "x", x, (n, c), x), 0), _CHANNELS.pack(*_strided(where, "y", y, (n, c), x), 0),
                                _flat32(where, "weight", weight, c * taps, x), _flat32(where, "bias", bias, c, x), stream)
    if rc:
        raise BloadError(rc, where)


SCAN_RUN = 16


def bload_scan_buffers(pos, x, a, gradient: bool = True, carry: bool | None = None):
    """(carry, work) for x [blocks, t_block, channels] and a [channels, states]: the float32 states that bload_scan keeps for the
    gradient, [blocks, ceil(t_block / 16), channels, states], and scratch: of bload_scan_grad, which serves both calls, or with
    gradient False of bload_scan alone, which needs less (None where none is needed).  carry: whether to make it (None: with
    gradient).  Calls that may overlap on the GPU need a scratch each."""
    b, t = pos.shape
    c, states = x.shape[-1], a.shape[-1]
    n = load().bload_scan_work_bytes(b, t, c, states, 1 if gradient else 0)
    return (x.new_empty((b, -(-t // SCAN_RUN), c, states), dtype=_torch()[2]) if (gradient if carry is None else carry) else None,
            x.new_empty(n, dtype=_torch()[5]) if n else None)


def _scan(where, pos, x, dt, a, b, c, d, dt_bias, z, softplus, carry, work, stream):
    """(packed fields up to z, of d_carry to work_bytes, stream)"""
    (blocks, t), code, stream = _begin(where, pos, x, 3, stream)
    channels = x.shape[2]
    if a.dim() != 2:
        raise ValueError("%s: a is [channels, states]" % where)
    states, shape = a.shape[1], (blocks, t, channels)
    rows = (blocks, t, states)
    return ((blocks, channels, t, code, states, 1 if softplus else 0, pos.data_ptr(), _flat32(where, "a", a, channels * states, x),
             _flat32(where, "d", d, channels, x), _flat32(where, "dt_bias", dt_bias, channels, x), *_strided(where, "x", x, shape, x),
             *_strided(where, "dt", dt, shape, x), *_strided(where, "b", b, rows, x), *_strided(where, "c", c, rows, x),
             *(_NONE3 if z is None else _strided(where, "z", z, shape, x))),
            (_flat32(where, "carry", carry, blocks * -(-t // SCAN_RUN) * channels * states, x), *_work(where, work, x)), stream)


def bload_scan(pos, x, dt, a, b, c, y, d=None, dt_bias=None, z=None, softplus: bool = True, carry=None, work=None, seq_id=None,
               last=None, stream=None) -> None:
    """Selective state-space scan inside the sequences of packed blocks: with delta = softplus(dt + dt_bias), per channel and state n
    h_s = exp(delta a[n]) h_{s-1} + delta b_s[n] x_s, y = sum_n c_s[n] h_s + d x, times z sigmoid(z) if z is given.  x, dt, y, z:
    [blocks, t_block, channels], b, c: [blocks, t_block, states] (float32, float16 or bfloat16, strided); a: float32 [channels,
    states], at most 64 states; d, dt_bias: float32 [channels] or None; softplus False: delta = dt + dt_bias.  carry, work from
    bload_scan_buffers (carry None: no gradient will be asked for).  last: float32 [sequences, channels, states] or None: the state
    behind every sequence of the batch, numbered by seq_id (int32 [blocks, t_block] from bload_pack), for bload_scan_step."""
    where = "bload_scan"
    head, kept, stream = _scan(where, pos, x, dt, a, b, c, d, dt_bias, z, softplus, carry, work, stream)
    rc = load().bload_scan(_SCAN.pack(*head, *_strided(where, "y", y, x.shape, x), *kept,
                                      *_sequences(where, pos, seq_id, last, "last", a.shape, _torch()[2]), *_NONE18, 0, 0, 0), stream)
    if rc:
        raise BloadError(rc, where)


def bload_scan_grad(pos, x, dt, a, b, c, carry, dy, dx, ddt, da, db, dc, d=None, dd=None, dt_bias=None, ddt_bias=None, z=None, dz=None,
                    softplus: bool = True, work=None, stream=None) -> None:
    """Gradients of bload_scan from dy, with the forward call's carry: dx, ddt, dz like x, db and dc like b, and summed over all frames da
    [channels, states], dd, ddt_bias [channels] (float32; the last two may be None: not wanted).  dz is needed where z is given."""
    where = "bload_scan_grad"
    head, kept, stream = _scan(where, pos, x, dt, a, b, c, d, dt_bias, z, softplus, carry, work, stream)
    channels = x.shape[2]
    if (z is None) != (dz is None):
        raise ValueError("%s: dz goes with z" % where)
    rc = load().bload_scan_grad(_SCAN.pack(
        *head, *_NONE3, *kept, 0, 0, 0, *_strided(where, "dy", dy, x.shape, x), *_strided(where, "dx", dx, x.shape, x),
        *_strided(where, "ddt", ddt, x.shape, x), *_strided(where, "db", db, b.shape, x), *_strided(where, "dc", dc, b.shape, x),
        *(_NONE3 if dz is None else _strided(where, "dz", dz, x.shape, x)), _flat32(where, "da", da, a.numel(), x),
        _flat32(where, "dd", dd, channels, x), _flat32(where, "ddt_bias", ddt_bias, channels, x)), stream)
    if rc:
        raise BloadError(rc, where)


def bload_scan_step(pos, state, x, dt, a, b, c, y, d=None, dt_bias=None, z=None, softplus: bool = True, next_state=None, stream=None) -> None:
    """bload_scan for one new frame of each of several sequences: x, dt, y, z [rows, channels], b, c [rows, states]; state: float32
    [rows, channels, states], moves on in place or into next_state.  pos as in bload_conv_step."""
    where = "bload_scan_step"
    n, channels, code, stream = _rows(where, pos, x, stream)
    if a.dim() != 2:
        raise ValueError("%s: a is [channels, states]" % where)
    states, f32 = a.shape[1], _torch()[2]
    shape = (n, channels, states)
    at = _state(where, "state", state, shape, f32, x)
    to = at if next_state is None else _state(where, "next_state", next_state, shape, f32, x)
    rows, narrow = (n, channels), (n, states)
    rc = load().bload_scan_step(_SCAN_STEP.pack(
        n, channels, code, states, 1 if softplus else 0, pos.data_ptr(), _flat32(where, "a", a, channels * states, x),
        _flat32(where, "d", d, channels, x), _flat32(where, "dt_bias", dt_bias, channels, x), at, to, *_strided(where, "x", x, rows, x), 0,
        *_strided(where, "dt", dt, rows, x), 0, *_strided(where, "b", b, narrow, x), 0, *_strided(where, "c", c, narrow, x), 0,
        *(_NONE3 if z is None else (*_strided(where, "z", z, rows, x), 0)), *_strided(where, "y", y, rows, x), 0), stream)
    if rc:
        raise BloadError(rc, where)


def bload_device_timeouts() -> int:
    """Bounded device-side waits of the layers' kernels that gave up on the current device (0 unless the hardware failed)."""
    return int(load().bload_device_timeouts())
