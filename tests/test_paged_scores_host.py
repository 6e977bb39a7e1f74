"""CPU-only checks of the weight that cached tokens gather: what its entry point refuses before anything is launched, and the plain form."""
import ctypes as C

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import paged_plain, scores_plain as plain

INV, UNS = -1, -2


def _t4(ptr=0x10000, dtype=zb.ZC_BF16, B=1, H=32, L=5, D=128):
    return zb.zc_tensor4(ptr, dtype, 0, B, H, L, D, H * L * D, L * D, D)


def test_refuses_bad_arguments_before_launch():
    lib = zb.load()

    def call(q=None, kp=None, table=0x30000, row=4, cols=4, start=0x40000, kv=0x50000, R=3, window=0, sinks=0, scale=0.0, lse=0x60000, decay=1.0,
             scores=0x70000):
        q, kp = q or _t4(), kp or _t4(B=10, H=8, L=16)
        return lib.zc_paged_scores(C.byref(q), C.byref(kp), table, row, cols, start, kv, R, window, sinks, scale, lse, decay, scores, None)
    nan = float("nan")
    for kw in (dict(table=None), dict(start=None), dict(kv=None), dict(lse=None), dict(scores=None), dict(scores=0x70008), dict(row=3), dict(cols=-1), dict(R=-1),
               dict(window=-1), dict(sinks=-1), dict(scale=-0.1), dict(scale=nan), dict(scale=3e38), dict(decay=-0.1), dict(decay=1.01), dict(decay=nan),
               dict(table=0x30002), dict(start=0x40001), dict(kv=0x50002), dict(lse=0x60002), dict(q=_t4(H=30)), dict(q=_t4(B=2)), dict(q=_t4(dtype=zb.ZC_F16)),
               dict(q=_t4(D=64)), dict(q=_t4(ptr=None)), dict(q=_t4(ptr=0x10004)), dict(kp=_t4(ptr=None, B=10, H=8, L=16))):
        assert call(**kw) == INV, kw
    for kw in (dict(R=1 << 24), dict(kp=_t4(B=10, H=8, L=24)), dict(q=_t4(L=1 << 26)), dict(cols=1 << 31, row=1 << 31), dict(kp=_t4(B=10, H=8, L=8))):
        assert call(**kw) == UNS, kw
    # nothing to do is no error, and needs no memory
    assert call(q=_t4(L=0, ptr=None), table=None, start=None, kv=None, lse=None) == 0
    assert call(R=0, table=None, start=None, kv=None, lse=None) == 0 and call(cols=0, table=None) == 0


def test_binding_refuses_tensors_that_are_not_what_a_call_needs():
    x, pages, i = torch.zeros(3, 2, 64), torch.zeros(4, 2, 16, 64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        zb.zc_paged_scores(x, pages, i[:, None], torch.zeros(4, dtype=torch.int32), i, torch.zeros(2, 3), torch.zeros(4, 2, 16))


def test_plain_weights_by_hand():
    p = paged_plain.Pages([2], [3], 2, 1, 64, torch.float32, device="cpu", seed=1)
    lse = plain.normalisers(p)
    got, off = plain.gathered(p, 0, lse, torch.tensor([[10.0, 20.0, 30.0]]), decay=0.5)
    a = torch.stack([torch.softmax((p.q[:, h].double() @ p.k[0][0].double().T / 8.0).masked_fill(torch.tensor([[False, False, True], [False] * 3]), -torch.inf), -1)
                     for h in range(2)])
    assert torch.allclose(got[0], a.sum((0, 1)) + torch.tensor([5.0, 0.0, 0.0], dtype=torch.float64), atol=1e-6)
    assert float(got.sum()) == pytest.approx(5.0 + 4.0, abs=1e-5) and float(off.max()) < 1e-4
