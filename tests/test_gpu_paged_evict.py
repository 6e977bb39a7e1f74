"""zc_paged_evict against lists and loops on the CPU: what stays, where it goes, which pages are left - whole numbers and copies, equal in every bit."""
import threading

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import evict_plain as plain

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"


class Cache:
    def __init__(self, kv_len, Hkv, D, dtype, page=16, by_head=True, seed=0, scores="random", cols=None, spare=3):
        g = torch.Generator().manual_seed(seed)
        have = [-(-max(n, 0) // page) for n in kv_len]
        N, cols = sum(have) + spare, cols or max(have + [1])
        order = torch.randperm(N, generator=g).int()
        self.table = torch.full((len(kv_len), cols), -9, dtype=torch.int32)
        at = 0
        for r, n in enumerate(have):
            self.table[r, :n] = order[at:at + n]
            at += n
        shape = (N, Hkv, page, D) if by_head else (N, page, Hkv, D)
        self.kp, self.vp = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
        if not by_head:
            self.kp, self.vp = self.kp.transpose(1, 2), self.vp.transpose(1, 2)
        x = torch.randn(N, Hkv, page, generator=g)
        self.sp = {"random": lambda: torch.exp(2 * x), "ties": lambda: (x * 2).round() / 4, "equal": lambda: torch.ones_like(x),
                   "zeros": lambda: torch.where(x > 0, 0.0, -0.0), "infinite": lambda: torch.where(x > 1, float("inf"), x)}[scores]().contiguous()
        self.kv_len, self.free = list(kv_len), torch.arange(100, 100 + 2 * N, dtype=torch.int32)

    def check(self, keep, most=None, sinks=0, recent=0, together=False, n_free=5, n_list=None):
        most = max(keep + [0]) if most is None else most
        R, H = len(self.kv_len), self.kp.shape[1]
        kept = torch.full((R, 1 if together else H, most), -5, dtype=torch.int32)
        free = self.free[:n_list]
        want = plain.evict(self.kp, self.vp, self.sp, self.table, self.kv_len, keep, most, sinks, recent, together, kept, free, n_free)
        i32 = dict(dtype=torch.int32, device=DEV)
        # (a copy keeps the strides of a dense tensor)
        kp, vp, sp, f = self.kp.to(DEV), self.vp.to(DEV), self.sp.to(DEV), free.to(DEV)
        assert kp.stride() == self.kp.stride()
        new_len, got_kept, n_freed = zb.zc_paged_evict(kp, vp, sp, self.table.to(DEV), torch.tensor(self.kv_len, **i32), torch.tensor(keep, **i32), most,
                                                       sinks=sinks, recent=recent, together=together, free_pages=f,
                                                       n_free=torch.tensor([n_free], **i32), kept=kept.to(DEV))
        torch.cuda.synchronize()
        assert new_len.tolist() == want[3].tolist()
        assert int(n_freed) == want[6]
        assert torch.equal(f.cpu(), want[5])
        assert torch.equal(got_kept.cpu(), want[4])
        for got, x in ((kp, want[0]), (vp, want[1]), (sp, want[2])):
            same = got.cpu().view(torch.int16 if got.element_size() == 2 else torch.int32) == x.view(torch.int16 if x.element_size() == 2 else torch.int32)
            assert bool(same.all()), (~same).nonzero()[0].tolist()


@pytest.mark.parametrize("dtype,D,H,page,by_head", [(BF, 128, 2, 16, True), (HF, 64, 3, 32, False), (FL, 64, 1, 64, True), (FL, 128, 2, 16, False), (BF, 64, 5, 128, True)])
@pytest.mark.parametrize("together", [False, True])
def test_ragged_requests(dtype, D, H, page, by_head, together):
    c = Cache([300, 0, 1, 77, 64, 513, 16, 15], H, D, dtype, page, by_head)
    c.check([100, 5, 1, 70, 64, 37, 15, 0], sinks=4, recent=10, together=together)


@pytest.mark.parametrize("scores", ["ties", "equal", "zeros", "infinite"])
@pytest.mark.parametrize("together", [False, True])
def test_equal_scores_keep_the_first(scores, together):
    Cache([700, 200, 33], 2, 64, BF, scores=scores).check([300, 199, 32], sinks=1, recent=5, together=together)
    Cache([700, 200, 33], 2, 64, BF, scores=scores).check([300, 1, 2], together=together)


@pytest.mark.parametrize("sinks,recent", [(0, 0), (50, 0), (0, 50), (30, 40), (50, 50), (1000, 3), (3, 1000), (2 ** 31 - 1, 2 ** 31 - 1), (25, 25)])
def test_first_and_newest_tokens(sinks, recent):
    Cache([120, 50, 51, 400], 2, 64, HF).check([50] * 4, sinks=sinks, recent=recent)


@pytest.mark.parametrize("keep,most", [([0, 0, 0], 0), ([-3, 20, 2 ** 31 - 1], 40), ([1, 1, 1], 1), ([500, 500, 500], 500), ([99, 100, 101], 200)])
def test_budgets(keep, most):
    Cache([100, 100, 100], 2, 64, BF).check(keep, most=most, recent=7)


@pytest.mark.parametrize("kv,keep,scores", [(8192, 8191, "random"), (8193, 4000, "random"), (20000, 9000, "ties"), (24577, 1, "random"), (17000, 16384, "equal"), (32769, 9000, "ties"), (75000, 30000, "random")])
@pytest.mark.parametrize("together", [False, True])
def test_long_requests(kv, keep, scores, together):
    Cache([kv, 40], 1 if not together else 2, 64, BF, page=64, scores=scores).check([keep, 40], sinks=4, recent=keep // 3, together=together)


@pytest.mark.parametrize("kv", [1, 15, 1023, 1024, 1025, 2047, 2048, 2049, 4097])
@pytest.mark.parametrize("keep", [1, 63, 64, 65, 256, 257])
def test_sizes_of_workgroups(kv, keep):
    Cache([kv, max(kv - 7, 0), min(kv, 70)], 2, 128 if keep < 200 else 64, BF).check([keep, keep - 1, 33], sinks=2, recent=3, together=kv % 2 == 0)


def test_many_short_requests():
    n = [(37 * i) % 150 for i in range(300)]
    Cache(n, 3, 64, HF, page=32).check([k // 2 for k in n], recent=4)


def test_lists_that_pages_do_not_fit():
    c = Cache([300, 200, 100], 1, 64, BF)
    for n_free, n_list in ((0, 10), (5, 6), (5, 5), (40, 10), (-4, 20)):
        c.check([16, 17, 0], n_free=n_free, n_list=n_list)


def test_a_table_with_missing_pages_and_lengths_outside_it():
    c = Cache([300, 200], 2, 64, BF, spare=0)
    c.table[0, 3], c.table[0, 7], c.table[1, 1], c.table[1, 5] = -1, 10 ** 9, -2 ** 31, 2 ** 31 - 1
    c.kv_len = [10 ** 9, -7]
    c.check([150, 150], sinks=2, recent=30)
    c.kv_len = [300, 200]
    for together in (False, True):
        c.check([150, 150], sinks=2, recent=30, together=together)


def test_without_a_list_and_without_requests():
    c = Cache([300, 200], 2, 64, BF)
    i32 = dict(dtype=torch.int32, device=DEV)
    args = [x.to(DEV) for x in (c.kp, c.vp, c.sp, c.table)]
    new_len, kept, n_freed = zb.zc_paged_evict(*args, torch.tensor(c.kv_len, **i32), torch.tensor([20, 300], **i32), 300)
    assert new_len.tolist() == [20, 200] and n_freed is None and kept.shape == (2, 2, 300)
    none = torch.zeros(0, **i32)
    before = [x.clone() for x in args]
    _, _, n_freed = zb.zc_paged_evict(*args[:3], args[3][:0], none, none, 300, free_pages=torch.zeros(4, **i32), n_free=torch.zeros(1, **i32))
    assert int(n_freed) == 0 and all(torch.equal(x, y) for x, y in zip(args, before))


def test_a_captured_eviction_replays():
    """Two graphs with the choice of all heads, which needs a workspace, replayed by turns with eager calls between them."""
    caches = [Cache([900, 300], 3, 64, BF, seed=s) for s in (1, 2)]
    i32 = dict(dtype=torch.int32, device=DEV)
    states = []
    for c in caches:
        kept = torch.full((2, 1, 200), -5, dtype=torch.int32)
        want = plain.evict(c.kp, c.vp, c.sp, c.table, c.kv_len, [200, 100], 200, 2, 9, True, kept, c.free, 3)
        s = {"from": [x.to(DEV) for x in (c.kp, c.vp, c.sp, kept, c.free)], "want": want, "table": c.table.to(DEV),
             "kv": torch.tensor(c.kv_len, **i32), "keep": torch.tensor([200, 100], **i32), "n_free": torch.tensor([3], **i32),
             "new": torch.zeros(2, **i32), "freed": torch.zeros(1, **i32)}
        s["now"] = [x.clone() for x in s["from"]]
        states.append(s)

    def call(s):
        kp, vp, sp, kept, free = s["now"]
        zb.zc_paged_evict(kp, vp, sp, s["table"], s["kv"], s["keep"], 200, sinks=2, recent=9, together=True, free_pages=free, n_free=s["n_free"],
                          new_len=s["new"], kept=kept, n_freed=s["freed"])

    def check(s):
        torch.cuda.synchronize()
        for got, x in zip(s["now"], (*s["want"][:3], s["want"][4], s["want"][5])):
            assert torch.equal(got.cpu(), x)
        assert s["new"].tolist() == s["want"][3].tolist() and int(s["freed"]) == s["want"][6]

    def reset(s):
        for x, y in zip(s["now"], s["from"]):
            x.copy_(y)
        s["new"].zero_()
        s["freed"].zero_()
    graphs = []
    for s in states:
        reset(s)
        call(s)
        check(s)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call(s)
        graphs.append(g)
    for turn in range(4):
        for i in (0, 1):
            reset(states[i])
            reset(states[1 - i])
            call(states[1 - i])
            graphs[i].replay()
            check(states[i])
            check(states[1 - i])


def test_threads_that_share_a_stream():
    """Calls of two threads on the default stream, each with a workspace: their launches do not come between each other's."""
    i32 = dict(dtype=torch.int32, device=DEV)
    caches = [Cache([2000, 300], 3, 64, BF, seed=s) for s in (3, 4)]
    out = [None, None]

    def work(n):
        c = caches[n]
        results = []
        for _ in range(20):
            kp, vp, sp = (x.to(DEV) for x in (c.kp, c.vp, c.sp))
            new, kept, _ = zb.zc_paged_evict(kp, vp, sp, c.table.to(DEV), torch.tensor(c.kv_len, **i32), torch.tensor([500, 100], **i32), 500, together=True)
            results.append((kp, kept[0, :, :500], kept[1, :, :100]))
        out[n] = results
    threads = [threading.Thread(target=work, args=(n,)) for n in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for c, results in zip(caches, out):
        kept = torch.full((2, 1, 500), -5, dtype=torch.int32)
        want = plain.evict(c.kp, c.vp, c.sp, c.table, c.kv_len, [500, 100], 500, 0, 0, True, kept, c.free, 0)
        for kp, a, b in results:
            assert torch.equal(kp.cpu(), want[0]) and torch.equal(a.cpu(), want[4][0]) and torch.equal(b.cpu(), want[4][1, :, :100])
