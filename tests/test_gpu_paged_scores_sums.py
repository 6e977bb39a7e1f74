"""zc_paged_scores over many rows: the sum of a token's weights rounds by the rows of a tile and by the tiles, not by all rows one after the other."""
import math

import pytest
import torch

from tests import scores_plain as plain
from tests.test_gpu_paged_scores import BF, DEV, FL, HF, Step

pytestmark = pytest.mark.gpu


def check(q_len, kv_len, Hq, Hkv, D, dtype, inverse, adds, **kw):
    """Rows of zeros: every weight is 1 / inverse, whatever the keys.  adds: additions that a request's sums go through, one after the other."""
    s = Step(q_len, kv_len, Hq, Hkv, D, dtype, **kw)
    p = s.p
    p.q.zero_()
    s.lse = torch.full((Hq, p.T), math.log(inverse), dtype=torch.float32, device=DEV)
    s.scores.zero_()
    got = s.scores.clone()
    s.call(got)
    torch.cuda.synchronize()
    n = float(s.lse[0, 0])
    for r, nq in enumerate(q_len):
        if nq == 0:
            continue
        now, _ = s.at(got, r)
        rows = plain.seen(kv_len[r], nq, 0, 0, DEV).sum(0).double() * (Hq // Hkv)
        want = (rows * math.exp(-n))[None].expand_as(now)
        # the change to base 2: 2^-24 of the logarithm for its product and for the constant; the exponential by 2^-22; every addition by 2^-24
        off = want * (2.0 ** -23 * abs(n) + 2.0 ** -22 + adds(nq * Hq // Hkv) * 2.0 ** -24)
        assert bool(((now.double() - want).abs() <= off).all()), (r, ((now.double() - want) / want * 2.0 ** 24).abs().max().item())


@pytest.mark.parametrize("inverse", [1.7, 3.3, 5.0])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (FL, 64), (FL, 128)])
@pytest.mark.parametrize("nq,kv,Hkv", [(2000, 2100, 1), (1500, 6000, 8)])       # (tiles of 64 keys, and of 128)
def test_chunks(dtype, D, nq, kv, Hkv, inverse):
    # a lane has a quarter of 256 rows (fp32: of 64), adds these up and then what all such parts gave; then the rest, products, lanes and waves, and the score
    part = 64 if dtype == FL else 256
    check([nq], [kv], 5 * Hkv, Hkv, D, dtype, inverse, lambda rows: part / 4 + rows / part + 5)


@pytest.mark.parametrize("inverse", [1.7, 3.3, 5.0])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (FL, 64), (FL, 128)])
def test_chunks_among_requests_without_tokens(dtype, D, inverse):
    # a lane has 16 of 32 rows
    check([120, 1] + [0] * 200, [500, 40] + [5] * 200, 64, 2, D, dtype, inverse, lambda rows: 16 + rows / 32 + 3)
