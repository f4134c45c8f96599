"""Which forward scans are cut into segments (they need scratch) and which walk every block in one piece (they need none); host only."""
import pytest

import paper_2310_10879_b200 as B


def scratch(blocks, t, groups, gradient=0, states=16):
    """of `blocks` * `groups` walks"""
    return B.load().bload_scan_work_bytes(blocks, t, groups * 64, states, gradient)


@pytest.mark.parametrize("blocks,groups", [(1, 149), (5, 32), (6, 32), (1, 221)])
def test_long_blocks_of_less_than_three_quarters_of_a_wave_are_cut(blocks, groups):
    for t in (2048, 4096, 32768):
        assert scratch(blocks, t, groups) > 0 and scratch(blocks, t, groups, 1) > 0, t


@pytest.mark.parametrize("blocks,groups", [(6, 37), (8, 30), (8, 32), (8, 37)])
def test_three_quarters_of_a_wave_or_more_walk_in_one_piece(blocks, groups):
    for t in (200, 1024, 4096, 32768):
        assert scratch(blocks, t, groups) == 0, t


def test_shorter_blocks_are_cut_for_fewer_walks():
    for t in (16, 203, 512, 767 - 15):
        assert scratch(1, t, 149) == 0 and scratch(5, t, 32) == 0, t
    for t in (768, 1024, 2032):
        assert scratch(6, t, 32) > 0 and scratch(1, t, 198) == 0, t
