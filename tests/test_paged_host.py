"""CPU-only checks of the paged cache: what its entry points refuse before anything is launched, and the plain forms the GPU
tests compare with."""
import ctypes as C

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import paged_plain as plain

INV, UNS, WSP = -1, -2, -3


def _t4(ptr=0x1000, dtype=zb.ZC_BF16, B=1, H=8, L=64, D=128):
    return zb.zc_tensor4(ptr, dtype, 0, B, H, L, D, H * L * D, L * D, D)


def test_tables_refuse_bad_arguments_before_launch():
    lib = zb.load()

    def call(q=0x1000, kv=0x2000, R=4, table=0x3000, row=8, cols=8, free=0x4000, n=16, n_free=0x5000, page=16, start=0x6000, slots=0x7000, T=9, taken=0x8000):
        return lib.zc_paged_tables(q, kv, R, table, row, cols, free, n, n_free, page, start, slots, T, taken, None)
    for kw in (dict(q=None), dict(kv=None), dict(table=None), dict(start=None), dict(slots=None), dict(taken=None), dict(free=None), dict(R=-1), dict(T=-1),
               dict(n=-1), dict(cols=-1), dict(row=7), dict(q=0x1002), dict(n_free=0x5001), dict(slots=0x7003), dict(table=0x3001)):
        assert call(**kw) == INV, kw
    for kw in (dict(page=0), dict(page=8), dict(page=24), dict(page=-16), dict(page=131072), dict(page=1 << 40), dict(R=1 << 31), dict(T=1 << 31), dict(n=1 << 31),
               dict(cols=1 << 31, row=1 << 31)):
        assert call(**kw) == UNS, kw


def test_store_and_load_refuse_bad_arguments_before_launch():
    lib = zb.load()
    pages = dict(B=10, H=8, L=16)

    def store(k=None, v=None, slots=0x3000, kp=None, vp=None):
        k, v, kp, vp = (x or y for x, y in ((k, _t4()), (v, _t4()), (kp, _t4(**pages)), (vp, _t4(**pages))))
        return lib.zc_paged_store(C.byref(k), C.byref(v), slots, C.byref(kp), C.byref(vp), None)

    def load(k=None, v=None, table=0x3000, row=4, cols=4, kv=0x4000, kp=None, vp=None):
        k, v, kp, vp = (x or y for x, y in ((k, _t4(B=3)), (v, _t4(B=3)), (kp, _t4(**pages)), (vp, _t4(**pages))))
        return lib.zc_paged_load(C.byref(kp), C.byref(vp), table, row, cols, kv, C.byref(k), C.byref(v), None)
    assert store(slots=None) == INV and store(slots=0x3002) == INV
    assert store(k=_t4(B=2)) == INV and store(k=_t4(H=4)) == INV and store(v=_t4(L=63)) == INV and store(k=_t4(dtype=zb.ZC_F16)) == INV
    assert store(k=_t4(ptr=0x1008)) == INV and store(k=_t4(D=64)) == INV and store(k=_t4(ptr=None)) == INV
    assert load(table=None) == INV and load(kv=None) == INV and load(row=3) == INV and load(cols=-1) == INV and load(kv=0x4001) == INV
    assert load(k=_t4(B=2)) == INV and load(v=_t4(B=3, L=32)) == INV and load(v=_t4(B=3, dtype=zb.ZC_F16)) == INV and load(k=_t4(B=3, H=4)) == INV
    assert load(k=_t4(B=40000), v=_t4(B=40000)) == UNS and load(k=_t4(B=3, L=1 << 29), v=_t4(B=3, L=1 << 29)) == UNS
    for call in (store, load):
        assert call(vp=_t4(B=9, H=8, L=16)) == INV and call(vp=_t4(B=10, H=8, L=32)) == INV and call(vp=_t4(dtype=zb.ZC_F32, **pages)) == INV
        for L in (8, 17, 48, 131072):
            assert call(kp=_t4(B=10, L=L), vp=_t4(B=10, L=L)) == UNS
        assert call(kp=_t4(B=1 << 27, L=16), vp=_t4(B=1 << 27, L=16)) == UNS                # slots of more than 31 bits
        assert call(kp=_t4(D=96, **pages), vp=_t4(D=96, **pages)) == UNS
        wide = _t4(**pages)
        wide.sL = 1 << 27
        assert call(kp=wide) == UNS                                                         # rows too far apart for 32-bit offsets
        wide = _t4(**pages)
        wide.sB = 1 << 31
        assert call(vp=wide) == UNS                                                         # and pages
    # nothing to do is no error, and needs no memory
    assert store(k=_t4(ptr=None, L=0), v=_t4(ptr=None, L=0), slots=None) == 0
    assert load(k=_t4(ptr=None, B=0), v=_t4(ptr=None, B=0), table=None, kv=None) == 0
    assert load(k=_t4(B=3, L=0), v=_t4(B=3, L=0)) == 0


def test_attention_refuses_bad_arguments_before_launch():
    lib = zb.load()
    pages = dict(B=10, H=8, L=16)
    ws = 1 << 30

    def call(q=None, kp=None, vp=None, table=0x3000, row=4, cols=4, start=0x4000, kv=0x5000, R=3, window=0, sinks=0, scale=0.0, out=None, lse=0x6000, w=0x7000, wn=ws):
        q, kp, vp, out = (x or y for x, y in ((q, _t4(H=32, L=5)), (kp, _t4(**pages)), (vp, _t4(**pages)), (out, _t4(H=32, L=5))))
        return lib.zc_paged_attention(C.byref(q), C.byref(kp), C.byref(vp), table, row, cols, start, kv, R, window, sinks, scale, C.byref(out), lse, w, wn, None)
    for kw in (dict(table=None), dict(start=None), dict(kv=None), dict(row=3), dict(cols=-1), dict(R=-1), dict(window=-1), dict(sinks=-1), dict(scale=-0.1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(table=0x3001), dict(lse=0x6002), dict(start=0x4002), dict(q=_t4(H=30, L=5), out=_t4(H=30, L=5)),
               dict(q=_t4(H=32, L=6)), dict(out=_t4(H=8, L=5)), dict(q=_t4(B=2, H=32, L=5)), dict(q=_t4(H=32, L=5, dtype=zb.ZC_F16)), dict(out=_t4(H=32, L=5, D=64)),
               dict(out=_t4(H=32, L=5, ptr=None)), dict(vp=_t4(B=9, H=8, L=16)), dict(q=_t4(H=32, L=5, ptr=0x1004))):
        assert call(**kw) == INV, kw
    for kw in (dict(R=1 << 24), dict(kp=_t4(B=10, L=24), vp=_t4(B=10, L=24)), dict(q=_t4(H=32, L=1 << 26), out=_t4(H=32, L=1 << 26)), dict(cols=1 << 31, row=1 << 31)):
        assert call(**kw) == UNS, kw
    need = lib.zc_paged_attention_workspace(3, 5, 32, 8, 128)
    assert need > 0 and call(w=None) == WSP and call(wn=need - 1) == WSP and call(w=0x7008) == WSP
    assert call(q=_t4(H=32, L=0, ptr=None), out=_t4(H=32, L=0, ptr=None), w=None) == 0 and call(R=0, start=None, kv=None, table=None, w=None) == 0
    assert lib.zc_paged_attention_workspace(0, 5, 32, 8, 128) == lib.zc_paged_attention_workspace(3, 0, 32, 8, 128) == 0
    assert lib.zc_paged_attention_workspace(3, 5, 30, 8, 128) == 0


def test_binding_refuses_tensors_that_are_not_what_a_call_needs():
    """Tensors of the CPU never reach a launch."""
    x, pages = torch.zeros(3, 2, 64), torch.zeros(4, 2, 16, 64)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        zb.zc_paged_store(x, x, i, pages, pages)
    with pytest.raises(ValueError):
        zb.zc_paged_load(pages, pages, i[:, None], i)
    with pytest.raises(ValueError):
        zb.zc_paged_attention(x, pages, pages, i[:, None], torch.zeros(4, dtype=torch.int32), i)
    with pytest.raises(ValueError):
        zb.zc_paged_tables(i, i, i[:, None], i, 16, 3)


def test_plain_tables_by_hand():
    # 3 tokens of 20 are new: one page more is needed; a fresh request of 17: two
    table, start, slots, taken = plain.tables([3, 17], [20, 17], [[5, -1], [-1, -1]], [7, 8, 9], 3, 16, 22)
    assert table == [[5, -1], [9, 8]] or table == [[5, 9], [8, 7]]
    assert taken == 2 + (20 > 32) and start == [0, 3, 20]
    # (17 tokens were there: they had two pages, the second's entry is what it was)
    assert table == [[5, -1], [9, 8]] and slots == [-1, -1, -1] + [9 * 16 + j for j in range(16)] + [8 * 16] + [-1, -1]


def test_plain_attention_by_hand():
    p = plain.Pages([2], [3], 1, 1, 64, torch.float32, device="cpu", seed=1)
    o, lse, _, _ = p.want()
    x = (p.q[:, 0].double() @ p.k[0][0].double().T) / 8.0
    assert torch.allclose(o[0, 0], torch.softmax(x[0, :2], -1) @ p.v[0][0, :2].double()) and torch.allclose(lse[0, 1], torch.logsumexp(x[1], -1))
    o, lse, _, _ = p.want(window=1)
    assert torch.allclose(o[1, 0], p.v[0][0, 2].double()) and torch.allclose(lse[0, 0], x[0, 1])
    o, _, _, _ = p.want(window=1, sinks=1)
    assert torch.allclose(o[1, 0], torch.softmax(x[1, [0, 2]], -1) @ p.v[0][0, [0, 2]].double())
    p = plain.Pages([3], [1], 1, 1, 64, torch.float32, device="cpu")
    o, lse, _, _ = p.want()
    assert lse[0].tolist()[:2] == [-float("inf")] * 2 and torch.allclose(o[2, 0], p.v[0][0, 0].double()) and not o[:2].any()
