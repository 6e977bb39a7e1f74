"""CPU-only checks of the paged cache: which strides of outputs, scales and sizes are refused before anything is launched, and which are not."""
import ctypes as C

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests.test_paged_host import INV, UNS, WSP, _t4


def _strided(t, **kw):
    for name, value in kw.items():
        setattr(t, name, value)
    return t


OVERLAPS = [dict(sH=0), dict(sB=0), dict(sH=128, sL=128), dict(sH=64 * 128 - 8), dict(sB=64 * 128, sH=64 * 128), dict(sL=8 * 120, sH=128)]
APART = [dict(), dict(sL=8 * 128, sH=128), dict(sB=64 * 128, sH=10 * 64 * 128), dict(sL=256, sH=128 * 128, sB=8 * 128 * 128), dict(sL=17 * 128, sH=2 * 128, sB=64 * 17 * 128)]


@pytest.mark.parametrize("strides", OVERLAPS)
def test_outputs_whose_rows_overlap_are_refused(strides):
    lib = zb.load()
    x, pages, read = _t4(H=8, L=64), _t4(B=10), _t4(B=10, H=8)
    wrong = _strided(_t4(B=10), **strides)
    for kp, vp in ((wrong, pages), (pages, wrong)):
        assert lib.zc_paged_store(C.byref(x), C.byref(x), 0x3000, C.byref(kp), C.byref(vp), None) == INV
    for k, v in ((wrong, read), (read, wrong)):
        assert lib.zc_paged_load(C.byref(pages), C.byref(pages), 0x3000, 4, 4, 0x4000, C.byref(k), C.byref(v), None) == INV
    if "sB" in strides:                                                       # (a step's rows have one batch element)
        return
    q, out = _t4(H=8, L=64), _strided(_t4(H=8, L=64), sB=0, **strides)
    assert lib.zc_paged_attention(C.byref(q), C.byref(pages), C.byref(pages), 0x3000, 4, 4, 0x4000, 0x5000, 3, 0, 0, 0.0, C.byref(out), 0x6000, 0x7000, 1 << 30,
                                  None) == INV


@pytest.mark.parametrize("strides", APART)
def test_outputs_whose_rows_lie_apart_are_taken(strides):
    """(without a GPU a call that passes its checks ends at its launch)"""
    if torch.cuda.is_available():
        pytest.skip("the addresses are no memory")
    lib = zb.load()
    x, read = _t4(H=8, L=64), _t4(B=10)
    pages = _strided(_t4(B=10), **strides)
    assert lib.zc_paged_store(C.byref(x), C.byref(x), 0x3000, C.byref(pages), C.byref(pages), None) not in (INV, UNS, 0)
    assert lib.zc_paged_load(C.byref(read), C.byref(read), 0x3000, 4, 4, 0x4000, C.byref(pages), C.byref(pages), None) not in (INV, UNS, 0)
    out, q = _strided(_t4(H=8, L=64), **{**strides, "sB": 0}), _strided(_t4(H=8, L=64), sH=0)          # (what is read may overlap)
    assert lib.zc_paged_attention(C.byref(q), C.byref(read), C.byref(read), 0x3000, 4, 4, 0x4000, 0x5000, 3, 0, 0, 0.0, C.byref(out), 0x6000, 0x7000, 1 << 30,
                                  None) not in (INV, UNS, WSP, 0)


@pytest.mark.parametrize("scale,taken", [(2.3e38, True), (2.4e38, False), (3.3e38, False), (float("inf"), False), (1e-45, True)])
def test_scales_whose_logits_have_no_finite_factor_are_refused(scale, taken):
    if torch.cuda.is_available():
        pytest.skip("the addresses are no memory")
    q, pages = _t4(H=8, L=64), _t4(B=10)
    rc = zb.load().zc_paged_attention(C.byref(q), C.byref(pages), C.byref(pages), 0x3000, 4, 4, 0x4000, 0x5000, 3, 0, 0, scale, C.byref(q), 0x6000, 0x7000, 1 << 30, None)
    assert rc not in (INV, UNS, WSP, 0) if taken else rc == INV


@pytest.mark.parametrize("L,dtype,taken", [(1 << 28, zb.ZC_F32, False), ((1 << 28) - 16, zb.ZC_F32, True), (1 << 28, zb.ZC_BF16, True)])
def test_a_load_that_one_launch_cannot_count_is_refused(L, dtype, taken):
    if torch.cuda.is_available():
        pytest.skip("the addresses are no memory")
    pages, k = _t4(B=10, dtype=dtype), _t4(B=1, H=1, L=L, dtype=dtype)
    pages.H, pages.sH = 1, 0
    rc = zb.load().zc_paged_load(C.byref(pages), C.byref(pages), 0x3000, 1 << 22, 1 << 22, 0x4000, C.byref(k), C.byref(k), None)
    assert rc not in (INV, UNS, 0) if taken else rc == UNS
