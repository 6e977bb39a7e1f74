"""zc_paged_scores of fp32 chunks over many keys: every call gives the same bits.  Its waves pass each other by up to a tile of rows, and weigh a tile's
last products when the next tile's normalisers are there already."""
import pytest
import torch

from tests.test_gpu_paged_scores import BF, FL, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,Hq", [(FL, 64, 16), (FL, 128, 16), (FL, 64, 8), (BF, 128, 32)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1700, 70)])
def test_equal_calls_over_many_keys(dtype, D, Hq, window, sinks):
    """340 tiles of 128 keys and more of all heads (so that a wave's products are of two sets of keys), single tokens and short chunks beside the
    chunks on a CU, so that its waves run unevenly; of the chunks some have rows that not all see all keys and some have none of these."""
    s = Step([1, 300, 40, 0, 70, 129, 1, 1, 3], [900, 3000, 2500, 40, 2500, 700, 2000, 64, 700], Hq, 8, D, dtype, page=32, pad=3, window=window, sinks=sinks, decay=0.9)
    first = None
    for _ in range(12):
        got = s.scores.clone()
        s.call(got)
        if first is None:
            s.check(got)
            first = got
        assert torch.equal(got.nan_to_num(-1.0), first.nan_to_num(-1.0))
