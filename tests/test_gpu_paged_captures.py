"""Paged attention in graphs that were captured through HIP itself, which torch's allocator does not know of."""
import ctypes as C

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import paged_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, FL = torch.bfloat16, torch.float32


def _hip():
    """The HIP runtime of this process."""
    torch.cuda.synchronize()
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64.so" in line)
    lib = C.CDLL(path)
    P = C.c_void_p
    for name, args in (("hipStreamBeginCapture", [P, C.c_int]), ("hipStreamEndCapture", [P, C.POINTER(P)]),
                       ("hipGraphInstantiate", [C.POINTER(P), P, P, P, C.c_size_t]), ("hipGraphLaunch", [P, P]),
                       ("hipGraphExecDestroy", [P]), ("hipGraphDestroy", [P])):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = args
    return lib


def test_a_capture_of_hip_s_own_keeps_its_workspace():
    hip = _hip()
    # calls that are split; the third needs more memory than the first two
    ps = [plain.Pages([1], [6000], 8, 2, 64, BF, seed=50), plain.Pages([1, 1], [5000, 300], 8, 2, 64, BF, seed=51),
          plain.Pages([1, 90], [7000, 400], 8, 2, 128, FL, seed=52)]
    outs = [(torch.zeros_like(p.q), torch.zeros(8, p.T, dtype=torch.float32, device=DEV)) for p in ps]

    def call(i):
        p = ps[i]
        zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=outs[i][0], lse=outs[i][1])
    want = []
    for i, p in enumerate(ps):
        call(i)
        p.check(*outs[i])
        want.append([x.clone() for x in outs[i]])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = []
    for calls in ((0, 1), (1,), (0, 2, 0)):
        graph, run = C.c_void_p(), C.c_void_p()
        assert hip.hipStreamBeginCapture(side.cuda_stream, 2) == 0
        with torch.cuda.stream(side):
            for i in calls:
                call(i)
        assert hip.hipStreamEndCapture(side.cuda_stream, C.byref(graph)) == 0
        assert hip.hipGraphInstantiate(C.byref(run), graph, None, None, 0) == 0
        graphs.append((calls, graph, run))
    # whoever asks next has other memory: tensors of every size of workspace, on the stream of the captures
    with torch.cuda.stream(side):
        sizes = [zb.load().zc_paged_attention_workspace(len(p.q_len), p.T, 8, 2, p.D) for p in ps]
        others = [torch.full((n,), 0x5A, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(4)]
    torch.cuda.synchronize()
    for _ in range(4):
        for calls, _, run in graphs:
            for o, n in outs:
                o.zero_()
                n.zero_()
            torch.cuda.synchronize()
            assert hip.hipGraphLaunch(run, side.cuda_stream) == 0
            torch.cuda.synchronize()
            for i in calls:
                assert torch.equal(outs[i][0], want[i][0]) and torch.equal(outs[i][1], want[i][1])
            assert all(bool((x == 0x5A).all()) for x in others)
    for _, graph, run in graphs:
        assert hip.hipGraphExecDestroy(run) == 0 and hip.hipGraphDestroy(graph) == 0


def test_a_capture_of_torch_s_holds_no_memory_behind_its_graph():
    p = plain.Pages([1], [6000], 32, 8, 128, BF, seed=53)
    out, lse = torch.zeros_like(p.q), torch.zeros(32, 1, dtype=torch.float32, device=DEV)
    need = zb.load().zc_paged_attention_workspace(1, 1, 32, 8, 128)
    assert need > 1 << 20

    def capture():
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(10):                                               # (one after the other: one workspace)
                zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=out, lse=lse)
        g.replay()
        torch.cuda.synchronize()
        p.check(out, lse)
    capture()
    before = torch.cuda.memory_allocated()
    for _ in range(5):
        capture()
    assert torch.cuda.memory_allocated() - before < need


def test_captures_of_both_kinds_one_after_the_other():
    """A graph of torch's, one of HIP's own, one of torch's again: what each has for a workspace is asked for each capture."""
    hip = _hip()
    p = plain.Pages([1], [6000], 8, 2, 128, BF, seed=54)
    out, lse = torch.zeros_like(p.q), torch.zeros(8, 1, dtype=torch.float32, device=DEV)
    side = torch.cuda.Stream()

    def call():
        zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=out, lse=lse)
    need = zb.load().zc_paged_attention_workspace(1, 1, 8, 2, 128)
    torch.cuda.synchronize()
    replays, others, held = [], [], []
    for kind in ("torch", "hip", "torch", "hip"):
        if kind == "torch":
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call()
            replays.append(g.replay)
            held.append(g)
        else:
            graph, run = C.c_void_p(), C.c_void_p()
            assert hip.hipStreamBeginCapture(side.cuda_stream, 2) == 0
            with torch.cuda.stream(side):
                call()
            assert hip.hipStreamEndCapture(side.cuda_stream, C.byref(graph)) == 0
            assert hip.hipGraphInstantiate(C.byref(run), graph, None, None, 0) == 0
            replays.append(lambda run=run: hip.hipGraphLaunch(run, side.cuda_stream))
            held.append((graph, run))
        with torch.cuda.stream(side):
            others += [torch.full((need,), 0x5A, dtype=torch.uint8, device=DEV) for _ in range(3)]
        torch.cuda.synchronize()
    for _ in range(3):
        for replay in replays:
            out.zero_()
            lse.zero_()
            torch.cuda.synchronize()
            replay()
            torch.cuda.synchronize()
            p.check(out, lse)
            assert all(bool((x == 0x5A).all()) for x in others)
    for graph, run in (x for x in held if isinstance(x, tuple)):
        assert hip.hipGraphExecDestroy(run) == 0 and hip.hipGraphDestroy(graph) == 0
