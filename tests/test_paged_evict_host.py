"""CPU-only checks of the eviction from a paged cache: what its entry point refuses before anything is launched, and the plain form."""
import ctypes as C

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import evict_plain as plain

INV, UNS, WSP = -1, -2, -3


def _pool(ptr=0x10000, dtype=zb.ZC_BF16, B=10, H=8, L=16, D=128, sH=None):
    return zb.zc_tensor4(ptr, dtype, 0, B, H, L, D, H * L * D, L * D if sH is None else sH, D)


def test_refuses_bad_arguments_before_launch():
    lib = zb.load()

    def call(kp=None, vp=None, scores=0x20000, table=0x30000, row=8, cols=8, kv=0x40000, keep=0x50000, R=4, most=20, sinks=0, recent=0, together=0,
             new=0x60000, kept=0x70000, free=0x80000, n_list=9, n_free=0x90000, n_freed=0xa0000, ws=0xb0000, wn=1 << 30):
        kp, vp = kp or _pool(), vp or _pool()
        return lib.zc_paged_evict(C.byref(kp), C.byref(vp), scores, table, row, cols, kv, keep, R, most, sinks, recent, together, new, kept, free, n_list,
                                  n_free, n_freed, ws, wn, None)
    for kw in (dict(scores=None), dict(scores=0x20008), dict(table=None), dict(row=7), dict(cols=-1), dict(kv=None), dict(keep=None), dict(R=-1), dict(most=-1),
               dict(sinks=-1), dict(recent=-1), dict(new=None), dict(kept=None), dict(n_list=-1), dict(n_free=None), dict(kv=0x40002), dict(keep=0x50001),
               dict(new=0x60002), dict(kept=0x70002), dict(free=0x80002), dict(n_free=0x90001), dict(n_freed=0xa0001), dict(n_freed=0x90000), dict(table=0x30002),
               dict(new=0x40000), dict(new=0x50000), dict(new=0x4000c), dict(kv=0x5fff4), dict(vp=_pool(B=9)), dict(vp=_pool(dtype=zb.ZC_F16)),
               dict(vp=_pool(L=32)), dict(kp=_pool(ptr=None)), dict(kp=_pool(ptr=0x10008)), dict(kp=_pool(sH=0)), dict(vp=_pool(sH=8 * 128))):
        assert call(**kw) == INV, kw
    for kw in (dict(R=65536), dict(most=1 << 31), dict(cols=1 << 28, row=1 << 28), dict(n_list=1 << 31), dict(kp=_pool(L=24), vp=_pool(L=24)),
               dict(kp=_pool(H=21846), vp=_pool(H=21846)), dict(kp=_pool(D=96), vp=_pool(D=96))):
        assert call(**kw) == UNS, kw
    size = lib.zc_paged_evict_workspace
    assert size(4, 8, 8, 16, 1) == 4 * 8 * 16 * 4 + 16 and size(4, 8, 8, 16, 0) == 4 * 8 * 4 and size(0, 8, 8, 16, 1) == 0
    for together in (0, 1):
        need = size(4, 8, 8, 16, together)
        for kw in (dict(ws=None), dict(wn=need - 1), dict(ws=0xb0008)):
            assert call(together=together, **kw) == WSP, kw
    # nothing to do is no error
    assert call(R=0, kv=None, keep=None, new=None, kept=None, table=None, free=None, n_free=None, n_freed=None, ws=None, wn=0) == 0


def test_binding_refuses_tensors_that_are_not_what_a_call_needs():
    pages, i = torch.zeros(4, 2, 16, 64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        zb.zc_paged_evict(pages, pages, torch.zeros(4, 2, 16), i[:, None], i, i, 5)


def test_plain_choice_by_hand():
    s = [5.0, 1.0, 4.0, 4.0, 0.0, 9.0, 2.0]
    assert plain.choose(s, 3, 0, 0) == [0, 2, 5] and plain.choose(s, 4, 0, 0) == [0, 2, 3, 5]
    assert plain.choose(s, 3, 0, 1) == [0, 5, 6] and plain.choose(s, 3, 2, 1) == [0, 1, 6] and plain.choose(s, 3, 9, 2) == [0, 5, 6]
    assert plain.choose(s, 3, 1, 5) == [4, 5, 6] and plain.choose(s, 9, 1, 1) == list(range(7)) and plain.choose(s, 0, 1, 1) == []


def test_plain_eviction_by_hand():
    kp = torch.arange(3 * 16.0).reshape(3, 1, 16, 1)
    table = torch.tensor([[2, 0]], dtype=torch.int32)
    sp = torch.zeros(3, 1, 16)
    sp[2, 0, 5] = 1.0
    sp[0, 0, 1] = 2.0                                                     # token 17
    out = plain.evict(kp, kp, sp, table, [20], [3], 3, 0, 1, False, torch.zeros(1, 1, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 1)
    assert out[4].tolist() == [[[5, 17, 19]]] and out[3].tolist() == [3] and out[6] == 1 and out[5].tolist() == [0, 0]
    assert out[0][2, 0, :3, 0].tolist() == [32 + 5, 1, 3] and out[0][2, 0, 3:].equal(kp[2, 0, 3:]) and out[0][:2].equal(kp[:2])
    assert out[2][2, 0, :3].tolist() == [1.0, 2.0, 0.0]
