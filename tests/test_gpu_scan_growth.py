"""bload_scan and its gradient where exponentials are larger than 32 bits hold: they count only where there is a state to multiply."""
import pytest
import torch

import layer_util as L
import state_space_util as S
from test_gpu_scan import F32, call, compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,c,n,blocks", [(64, 24, 8, [[1, 20, 30, -3, 10]]), (2560, 20, 16, [[128, 128, 1, 1000, 1303]]), (40, 2048, 5, [[17, 23]] * 5),
                                          (64, 2048, 4, [[30, 34]] * 10)])
def test_growth_at_a_start_multiplies_nothing(t, c, n, blocks):
    """exp(delta a) of 150 to 600 e-folds on the first frame of every sequence: one piece, segments, halves, many walks."""
    i = S.scan_inputs(len(blocks), t, c, n, F32, 21)
    pos = L.positions(t, blocks)
    i["dt"] = torch.where((pos == 0)[..., None], -150.0, 0.1 * i["dt"].abs())
    i["a"] = -torch.linspace(1.0, 4.0, c * n, device=L.DEV).reshape(c, n)
    i["dt_bias"] = None
    compare(call(pos, i, softplus=False), blocks, i, softplus=False)
