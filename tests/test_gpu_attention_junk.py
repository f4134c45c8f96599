"""Attention over batches in which frames hold infinities and NaN: what may see them shows them, all else is as if they
were not there."""
import math

import pytest
import torch

import layer_util as L
import paper_2310_10879_b200 as B
from test_gpu_attention import BF, FP, buffers, call, inputs, slopes_of

pytestmark = pytest.mark.gpu
DEV = L.DEV


def without(blocks, bad):
    """The packing with the sequences of `bad` ({(block, index)}) as padding."""
    return [[-n if n > 0 and (b, k) in bad else n for k, n in enumerate(here)] for b, here in enumerate(blocks)]


def slots(blocks, t, bad):
    """bool [blocks, t]: slots of the sequences of `bad`."""
    m = torch.zeros((len(blocks), t), dtype=torch.bool, device=DEV)
    for b, here in enumerate(blocks):
        s = 0
        for k, n in enumerate(here):
            m[b, s:s + abs(n)] |= (b, k) in bad
            s += abs(n)
    return m


def compare_clean(got, blocks, t, bad, q, k, v, dout, **how):
    """Everything outside the sequences of `bad`, against the definition of the batch without them."""
    torch.cuda.synchronize()
    here = ~slots(blocks, t, bad)
    zero = {n: x.masked_fill(~here[..., None, None], 0.0) for n, x in (("q", q), ("k", k), ("v", v), ("dout", dout))}
    val, tol = L.attention(without(blocks, bad), zero["q"], zero["k"], zero["v"], zero["dout"], **how)
    frame = ~torch.isinf(val["lse"])
    L.close(got["lse"][frame], val["lse"][frame], tol["lse"][frame], "lse")
    for n in ("out", "dq", "dk", "dv"):
        L.close(got[n][here], val[n][here], tol[n][here], n)


@pytest.mark.parametrize("d", [24, 64, 128])
@pytest.mark.parametrize("dtype", [BF, FP], ids=["bf16", "fp16"])
def test_walks_of_a_single_tile_end_in_order(dtype, d):
    """Every CTA meets junk in the only tile of its walk, call after call: its products and copies have to have ended
    before the next CTA takes its place."""
    t, nb, h, hk = 40, 300, 4, 2
    blocks = [[3, 1, 7, 2, 9, 4, 12, -2]] * nb
    bad = {(b, k) for b in range(nb) for k in (1, 4)}
    q, k, v, dout = inputs(nb, t, h, hk, d, dtype)
    for x in (q, k, v, dout):
        x[slots(blocks, t, bad)] = math.nan
    pos = L.positions(t, blocks)
    first = {n: x.clone() for n, x in call(pos, q, k, v, dout).items()}
    for _ in range(20):
        again = call(pos, q, k, v, dout)
        for n in first:
            assert torch.equal(first[n].nan_to_num(7.0), again[n].nan_to_num(7.0)), n
    assert B.bload_device_timeouts() == 0
    few = {n: x[:8] for n, x in first.items()}
    compare_clean(few, blocks[:8], t, {x for x in bad if x[0] < 8}, q[:8], k[:8], v[:8], dout[:8])
