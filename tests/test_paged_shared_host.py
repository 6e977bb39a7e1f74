"""CPU-only checks of the attention over shared prefixes: what its entry point refuses before anything is launched, and the plain form."""
import ctypes as C

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import shared_plain as plain

INV, UNS, WSP = -1, -2, -3


def _t4(ptr=0x10000, dtype=zb.ZC_BF16, B=1, H=32, L=5, D=128):
    return zb.zc_tensor4(ptr, dtype, 0, B, H, L, D, H * L * D, L * D, D)


def test_refuses_bad_arguments_before_launch():
    lib = zb.load()
    pages = dict(B=10, H=8, L=16)

    def call(q=None, kp=None, vp=None, pre=0x30000, pre_row=4, pre_cols=4, pre_len=0x40000, groups=0x50000, P=2, table=0x60000, row=4, cols=4, start=0x70000,
             kv=0x80000, R=3, scale=0.0, out=None, lse=0x90000, ws=0xa0000, wn=1 << 40):
        q, kp, vp, out = (x or y for x, y in ((q, _t4()), (kp, _t4(**pages)), (vp, _t4(**pages)), (out, _t4())))
        return lib.zc_paged_shared_attention(C.byref(q), C.byref(kp), C.byref(vp), pre, pre_row, pre_cols, pre_len, groups, P, table, row, cols, start, kv, R, scale,
                                             C.byref(out), lse, ws, wn, None)
    for kw in (dict(pre=None), dict(pre_len=None), dict(groups=None), dict(pre_row=3), dict(pre_cols=-1), dict(P=-1), dict(table=None), dict(start=None), dict(kv=None),
               dict(row=3), dict(cols=-1), dict(R=-1), dict(scale=-0.1), dict(scale=float("nan")), dict(scale=3e38), dict(pre=0x30001), dict(pre_len=0x40002),
               dict(groups=0x50003), dict(table=0x60001), dict(start=0x70002), dict(kv=0x80001), dict(lse=0x90002), dict(q=_t4(H=30), out=_t4(H=30)),
               dict(q=_t4(L=6)), dict(out=_t4(H=8)), dict(q=_t4(B=2)), dict(q=_t4(dtype=zb.ZC_F16)), dict(out=_t4(D=64)), dict(out=_t4(ptr=None)),
               dict(vp=_t4(B=9, H=8, L=16)), dict(q=_t4(ptr=0x10004))):
        assert call(**kw) == INV, kw
    for kw in (dict(P=1025), dict(R=1 << 24), dict(kp=_t4(B=10, L=24), vp=_t4(B=10, L=24)), dict(q=_t4(L=1 << 26), out=_t4(L=1 << 26)),
               dict(cols=1 << 31, row=1 << 31), dict(pre_cols=1 << 31, pre_row=1 << 31), dict(R=1 << 21, q=_t4(L=1 << 21), out=_t4(L=1 << 21))):
        assert call(**kw) == UNS, kw
    need = lib.zc_paged_shared_attention_workspace(2, 3, 5, 32, 8, 128)
    assert need > 0 and call(ws=None) == WSP and call(wn=need - 1) == WSP and call(ws=0xa0008) == WSP
    # without a prefix it is the paged attention, whose workspace it then needs
    none = lib.zc_paged_attention_workspace(3, 5, 32, 8, 128)
    assert lib.zc_paged_shared_attention_workspace(0, 3, 5, 32, 8, 128) == none <= need
    assert call(P=0, pre=None, pre_len=None, groups=None, wn=none - 1) == WSP and call(pre_cols=0, pre=None, wn=none - 1) == WSP
    # nothing to do is no error, and needs no memory
    assert call(q=_t4(L=0, ptr=None), out=_t4(L=0, ptr=None), ws=None) == 0 and call(R=0, start=None, kv=None, table=None, ws=None) == 0
    assert lib.zc_paged_shared_attention_workspace(2, 0, 5, 32, 8, 128) == lib.zc_paged_shared_attention_workspace(2, 3, 0, 32, 8, 128) == 0


def test_binding_refuses_tensors_that_are_not_what_a_call_needs():
    x, pages, i = torch.zeros(3, 2, 64), torch.zeros(4, 2, 16, 64), torch.zeros(3, dtype=torch.int32)
    j = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        zb.zc_paged_shared_attention(x, pages, pages, i[:, None], i, j, i[:, None], j, i)


def test_plain_attention_by_hand():
    s = plain.Shared([1, 2], [2, 2], [0, 1], [5], 2, 1, 64, torch.float32, device="cpu")
    o, lse, _, _, _ = s.want()
    p = s.p
    k, v = torch.cat([p.k[2][0], p.k[0][0]]).double(), torch.cat([p.v[2][0], p.v[0][0]]).double()
    x = p.q[0, 1].double() @ k.T / 8.0
    assert torch.allclose(o[0, 1], torch.softmax(x, 0) @ v) and torch.allclose(lse[1, 0], torch.logsumexp(x, 0))
    x = p.q[1, 0].double() @ p.k[1][0].double().T / 8.0                    # (no prefix, sees itself only)
    assert torch.allclose(o[1, 0], p.v[1][0, 0].double()) and torch.allclose(lse[0, 1], x[0])
