"""relay_attn_update_tables with more requests than a launch has wavefronts for at once (256 groups of 16)."""
import numpy as np
import pytest

from test_gpu_tables import _case, _check, _say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,bs,width,grow", [(4096, 16, 4, 9), (4097, 8, 5, 20), (5000, 16, 6, 33), (12345, 32, 3, 40)])
@pytest.mark.parametrize("supply", ["plenty", "scarce"])
def test_requests_that_a_wavefront_takes_in_turn(batch, bs, width, grow, supply):
    rng = np.random.Generator(np.random.PCG64(batch))
    want = batch * (grow // bs + 2)
    spare = want if supply == "plenty" else want // 6
    _say("batch %d block %d width %d grow %d spare %d" % (batch, bs, width, grow, spare))
    _check(*_case(rng, batch, bs, width, spare, grow), bs)
