"""Calls of two threads on one stream: what shares a stream's scratch memory is launched one call after the other."""
import ctypes as C
import threading
import time

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import paged_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def _together(*calls):
    """Runs the calls in a thread each, started at once; raises what one of them raised."""
    gate, errors = threading.Barrier(len(calls)), []

    def body(call):
        try:
            gate.wait()
            call()
        except BaseException as e:                                            # noqa: BLE001 (handed to the test's thread)
            errors.append(e)
    threads = [threading.Thread(target=body, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]


class _Counted:
    """Entry points that launch nothing and note how many calls were inside one at a time."""

    def __init__(self, *names):
        self.lib, self.names = zb.load(), names
        self.inside = self.most = self.calls = 0

    def _entry(self, *_):
        self.inside += 1
        self.calls += 1
        self.most = max(self.most, self.inside)
        time.sleep(0.002)                                                     # (the other thread runs meanwhile)
        self.inside -= 1
        return 0

    def __enter__(self):
        self.kept = [C.CFUNCTYPE(C.c_int, *getattr(self.lib, n).argtypes)(self._entry) for n in self.names]
        self._bind(dict(zip(self.names, self.kept)))
        return self

    def __exit__(self, *_):
        self._bind({})

    def _bind(self, instead):
        host = zb._native()
        host.bind(tuple(C.cast(instead.get(n) or getattr(self.lib, n), C.c_void_p).value for n in host.names()))


def _packed(B, H, D, n_hi, n_lo):
    slots = zb.load().zc_arena_slots
    return [zb.PackedTensor(B, H, D, slots(n_hi, 1), slots(n_lo, 1), 4, 2, s, lay, max_chunks=1)
            for s, lay in (("channel", zb.ZC_LAYOUT_ROW), ("cst", zb.ZC_LAYOUT_TGROUP))]


@pytest.mark.parametrize("kind", ["paged", "decode", "decode_static", "probe", "quantize", "quantize_kv"])
def test_calls_that_share_scratch_are_launched_one_at_a_time(kind):
    Q, K, V = (torch.randn(1, 4, 300, 64, device=DEV).to(BF) for _ in range(3))
    pos = torch.arange(200, 230, device=DEV, dtype=torch.int32)
    scores = torch.rand(1, 300, device=DEV)
    salient, regular = zb.zc_select_salient(scores, 100)
    Kp, Vp = _packed(1, 4, 64, 100, 200)
    zb.zc_quantize_pack_kv(K, V, salient, regular, Kp, Vp)
    p = plain.Pages([1], [3000], 4, 2, 64, BF, seed=1)
    names, call = {
        "paged": (["zc_paged_attention"], lambda: zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv)),
        "decode": (["zc_decode_attention"], lambda: zb.zc_decode_attention(Q[:, :, -1], Kp, Vp)),
        "decode_static": (["zc_decode_attention_static"], lambda: zb.zc_decode_attention_static(Q[:, :, -1], Kp, Vp, out=torch.empty(1, 4, 64, dtype=BF, device=DEV))),
        "probe": (["zc_probe_saliency", "zc_probe_accumulated"], lambda: (zb.zc_probe_saliency(Q, K, pos), zb.zc_probe_accumulated(Q, K, pos))),
        "quantize": (["zc_quantize_pack"], lambda: zb.zc_quantize_pack(K, salient, regular, Kp)),
        "quantize_kv": (["zc_quantize_pack_kv"], lambda: zb.zc_quantize_pack_kv(K, V, salient, regular, Kp, Vp))}[kind]
    torch.cuda.synchronize()
    with _Counted(*names) as c:
        _together(*([lambda: [call() for _ in range(5)]] * 3))
    assert c.calls == 15 * len(names) and c.most == 1


def test_two_threads_on_one_stream_split_and_join_their_own_rows():
    ps = [plain.Pages([1], [6000], 8, 2, 128, BF, seed=41), plain.Pages([1, 1, 40], [5000, 40, 333], 16, 8, 64, FL, seed=42)]
    want, outs = [], []
    for p in ps:
        o, n = torch.zeros_like(p.q), torch.zeros(p.Hq, p.T, dtype=torch.float32, device=DEV)
        zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=o, lse=n)
        p.check(o, n)
        want.append((o, n))
        outs.append([(torch.zeros_like(o), torch.zeros_like(n)) for _ in range(100)])
    torch.cuda.synchronize()

    def many(p, out):
        for o, n in out:
            zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=o, lse=n)
    _together(*(lambda p=p, o=o: many(p, o) for p, o in zip(ps, outs)))
    torch.cuda.synchronize()
    for (wo, wn), out in zip(want, outs):
        assert all(torch.equal(o, wo) and torch.equal(n, wn) for o, n in out)
