"""zc_paged_scores over rows that lie far apart: of one token to the next up to 4 GB."""
import pytest
import torch

from tests.test_gpu_paged_scores import BF, DEV, FL, HF, Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,mb", [(BF, 64, 128), (BF, 64, 132), (HF, 64, 144), (BF, 64, 255), (BF, 64, 256), (BF, 64, 270), (HF, 128, 255), (HF, 128, 257),
                                        (FL, 64, 255), (FL, 64, 257), (FL, 128, 260)])
def test_rows_far_apart(dtype, D, mb):
    """One head a group: 32 tokens (64 channels of 16 bits), 16 or 8 are requested with one base; their offsets pass 32 bits from 129, 257 MB a token on."""
    s = Step([140], [400], 1, 1, D, dtype)
    stride = (mb << 20) // dtype.itemsize
    store = torch.empty((s.p.T - 1) * stride + D, dtype=dtype, device=DEV)
    q = store.as_strided((s.p.T, 1, D), (stride, D, 1))
    q.copy_(s.p.q)
    got = s.scores.clone()
    s.call(got, q=q)
    torch.cuda.synchronize()
    s.check(got)
    del q, store
    torch.cuda.empty_cache()


def test_heads_far_apart():
    """Four heads a group, 1.1 GB from one to the next."""
    s = Step([70, 1], [300, 90], 4, 1, 64, BF)
    stride = 550 << 20
    store = torch.empty(3 * stride + s.p.T * 64, dtype=BF, device=DEV)
    q = store.as_strided((s.p.T, 4, 64), (64, stride, 1))
    q.copy_(s.p.q)
    got = s.scores.clone()
    s.call(got, q=q)
    torch.cuda.synchronize()
    s.check(got)
    del q, store
    torch.cuda.empty_cache()
