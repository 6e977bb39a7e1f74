"""Keys whose logits are -inf, in front of and between others: as if they were not there, to the accuracy of a call without them."""
import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import paged_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("q,kv,D,hidden", [
    (1, 4000, 64, [(0, 2000)]), (1, 4000, 128, [(0, 3999)]), (1, 5000, 64, [(64, 1500), (1501, 3000)]), (1, 300, 128, [(0, 40), (100, 164), (250, 251)]),
    (150, 4000, 64, [(0, 2000)]), (150, 4000, 128, [(0, 3850)]), (90, 300, 64, [(0, 40), (100, 164)]), (40, 1500, 128, [(31, 33), (500, 1400)])])
def test_keys_without_weight(q, kv, D, hidden, dtype):
    p = plain.Pages([q], [kv], 4, 2, D, dtype, seed=70 + kv + q)
    p.q[..., 1] = 1.0
    there = torch.ones(kv, dtype=torch.bool, device=DEV)
    for lo, hi in hidden:
        there[lo:hi] = False
        p.k[0][:, lo:hi, 1] = -float("inf")
    assert bool(there[kv - q:].all())                                         # (every row sees the same of them)
    p.write(0)
    out, lse = torch.full_like(p.q, 5.0), torch.full((4, p.T), 5.0, dtype=torch.float32, device=DEV)
    zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=out, lse=lse)
    # a weight of 0 and a part without a weight add exact zeros, so the bound is that of the request without these keys
    p.k, p.v = [p.k[0][:, there]], [p.v[0][:, there]]
    p.kv_len = [int(there.sum())]
    p.check(out, lse)
