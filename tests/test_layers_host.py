"""The host side of the layers on packed batches where no GPU is needed: what a call reads of its argument block, and
sizes that no batch has.  What would end the process if it were wrong runs in a process of its own, without a device."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def alone(code: str) -> int:
    """Exit code of `code`, run by a new interpreter that sees no device."""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="", PYTHONPATH=ROOT)
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    if done.returncode:
        print(done.stdout, done.stderr, file=sys.stderr)
    return done.returncode


BLOCK_AT_THE_END_OF_A_PAGE = """
import ctypes as C, mmap
from paper_2310_10879_b200 import _lib as E
L, P = E.load(), 1 << 20
libc = C.CDLL(None, use_errno=True)
page = mmap.PAGESIZE
pages = mmap.mmap(-1, 2 * page)
base = C.addressof(C.c_char.from_buffer(pages))
libc.mprotect.argtypes = [C.c_void_p, C.c_size_t, C.c_int]
assert libc.mprotect(base + page, page, 0) == 0  # nothing behind the first page may be touched
def at_the_end(block):
    C.memmove(base + page - len(block), block, len(block))
    return base + page - len(block)
heads = [P, 64 * 4 * 64, 4 * 64, 64]
attention = [2, 64, 4, 4, 64, E.BF16, 1, 0, 0.125, 0.0, 0, P, 0] + 4 * heads + [P]
rows = [P, 200 * 64, 64]
recurrence = [2, 64, 200, E.BF16, P] + 3 * rows + [P, P, 1 << 40] + 3 * rows
call = {
    "bload_attention": lambda: L.bload_attention(at_the_end(E._ATTENTION.pack(*attention)), None),
    "bload_attention_grad": lambda: L.bload_attention_grad(at_the_end(E._ATTENTION_GRAD.pack(*attention, *(4 * heads), P)), None),
    "bload_recurrence": lambda: L.bload_recurrence(at_the_end(E._RECURRENCE.pack(*recurrence)), None),
    "bload_recurrence_grad": lambda: L.bload_recurrence_grad(at_the_end(E._RECURRENCE.pack(*recurrence)), None),
    "bload_rotary": lambda: L.bload_rotary(P, 2, 64, 4, 64, E.BF16, at_the_end(E._HEADS.pack(*heads)), E._HEADS.pack(*heads), P, 64, 0, 1.0, None),
    "bload_rotary_grad": lambda: L.bload_rotary_grad(P, 2, 64, 4, 64, E.BF16, E._HEADS.pack(*heads), at_the_end(E._HEADS.pack(*heads)), P, 64, 0, 1.0, None),
}[NAME]
rc = call()
assert rc == E.ERR_CUDA, rc  # every argument was taken, and there is no device
"""


@pytest.mark.parametrize("name", ["bload_attention", "bload_attention_grad", "bload_recurrence", "bload_recurrence_grad",
                                  "bload_rotary", "bload_rotary_grad"])
def test_a_call_reads_nothing_behind_its_argument_block(name):
    assert alone("NAME = %r\n%s" % (name, BLOCK_AT_THE_END_OF_A_PAGE)) == 0


SIZES_WITHOUT_END = """
from paper_2310_10879_b200 import _lib as E
import ctypes as C
L, P = E.load(), 1 << 20
for blocks in (1, 1 << 20, (1 << 31) - 1, 1 << 31, 1 << 40, 1 << 58, (1 << 62) + 1, (1 << 63) - 1):
    for t in (1, 64, 65, 5000, E.MAX_T_BLOCK):
        for channels in (1, 64, 4096, (1 << 31) - 1, 1 << 31, 1 << 58, (1 << 63) - 1):
            parts = blocks * -(-channels // 64) * -(-t // 64)  # Python's integers have no end
            fits = blocks < 1 << 31 and channels < 1 << 31 and parts < 1 << 31
            need = L.bload_recurrence_work_bytes(blocks, t, channels)
            assert need < 1 << 42 and (fits or need == 0), (blocks, t, channels, need)
            a = E.RecurrenceArgs(blocks, channels, t, E.BF16, P)
            for n in ("gate", "x", "h", "dh", "dgate", "dx"):
                setattr(a, n, E.ChannelsTensor(P, 1 << 38, 1 << 38))
            a.d_carry, a.d_work, a.work_bytes = P, P, 1 << 60
            for call in (L.bload_recurrence, L.bload_recurrence_grad):
                rc = call(C.byref(a), None)
                assert rc == (E.ERR_CUDA if fits else E.ERR_ARG), (blocks, t, channels, rc)
"""


def test_sizes_whose_product_has_no_room_are_refused():
    """(In a process of its own: a wrong product once was a division by zero.)"""
    assert alone(SIZES_WITHOUT_END) == 0
