"""bload_scan and its gradient where forward and backward walk blocks in different pieces, with sequences that start at, just behind and
far from the edges of the pieces."""
import pytest
import torch

import layer_util as L
import state_space_util as S
import paper_2310_10879_b200 as B
from test_gpu_scan import BF, F32, FP, FRAMES, SUMS, call, compare

pytestmark = pytest.mark.gpu


def pieces(pos, i):
    """(forward in one piece, gradient's scratch in bytes)"""
    b, t = pos.shape
    c, n = i["a"].shape
    size = B.load().bload_scan_work_bytes
    return size(b, t, c, n, 0) == 0, size(b, t, c, n, 1)


def check(t, c, n, dtype, blocks, one_piece, gated):
    i = S.scan_inputs(len(blocks), t, c, n, dtype, 40, gated)
    pos = L.positions(t, blocks)
    assert pieces(pos, i)[0] == one_piece
    got = call(pos, i)
    compare(got, blocks, i)
    again = call(pos, i)
    torch.cuda.synchronize()
    for k in FRAMES + SUMS + ("carry",):
        if got[k] is not None:
            assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("dtype,c,n,gated", [(BF, 2048, 16, True), (F32, 2003, 7, False)])
def test_forward_in_one_piece_and_gradient_in_two(dtype, c, n, gated):
    """160 walks of 38 runs: the gradient's pieces meet at slot 304, or at the first start of the 152 slots behind it."""
    check(600, c, n, dtype, [[600], [304, 296], [305, 1, 294], [-303, 2, 295], [455, 145]], True, gated)
    check(600, c, n, dtype, [[456, 144], [300, -10, 290], [1] * 310 + [290], [310, -290], [-600]], True, gated)


@pytest.mark.parametrize("dtype,c,n", [(FP, 2048, 16), (BF, 1024, 32)])
def test_three_quarters_of_a_wave_of_longer_blocks(dtype, c, n):
    """256 walks of 50 runs: one piece forward, two in the gradient, which meet at slot 400 or in the 200 behind."""
    check(800, c, n, dtype, [[800], [400, 400], [401, 399], [599, 201], [600, 200], [-399, 401], [390, -20, 390], [16] * 50], True, False)


def test_walks_that_fill_a_wave_and_a_little_of_the_next():
    """600 walks of 50 runs: few segments both ways."""
    check(800, 64 * 120, 2, F32, [[800], [256, 272, 272], [257, 1, 270, 272], [383, 145, 272], [384, 416]], False, True)


def test_both_ways_in_segments_where_one_wave_is_partly_empty():
    """160 walks of 128 runs."""
    check(2048, 2048, 3, BF, [[2048], [1024, 1024], [700, 1, 1000, 347], [-100, 1900, -48], [513, 2, 1533]], False, True)
