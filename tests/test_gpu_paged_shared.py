"""zc_paged_shared_attention against float64, and against the paged attention where the prefix stands in every request's own pages."""
import math
import threading

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import shared_plain as plain

pytestmark = pytest.mark.gpu
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"


def run(s, sm_scale=0.0):
    p = s.p
    out, lse = torch.full_like(p.q, 7.0), torch.full((p.Hq, p.T), 7.0, dtype=torch.float32, device=DEV)
    zb.zc_paged_shared_attention(*s.args(), sm_scale=sm_scale, out=out, lse=lse)
    s.check(out, lse, sm_scale)
    assert bool((out[p.start[-1]:] == 7.0).all()) and bool((lse[:, p.start[-1]:] == 7.0).all()), "rows behind the last request"
    return out, lse


@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,by_head", [(BF, 128, 8, 2, 16, True), (HF, 64, 4, 4, 32, False), (FL, 64, 6, 2, 64, True), (FL, 128, 4, 1, 16, False),
                                                         (BF, 64, 8, 1, 128, True), (HF, 128, 3, 3, 16, True)])
def test_single_tokens_and_chunks(dtype, D, Hq, Hkv, page, by_head):
    run(plain.Shared([1] * 6, [9, 70, 1, 300, 64, 33], [0, 6], [500], Hq, Hkv, D, dtype, page=page, by_head=by_head, pad=3))
    run(plain.Shared([1, 40, 0, 90, 3, 1, 1, 5, 1], [30, 40, 10, 300, 3, 1, 200, 5, 17], [1, 4, 4, 7], [333, 90, 64], Hq, Hkv, D, dtype, page=page, by_head=by_head))


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 1000, 5000])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (FL, 64)])
def test_lengths_of_prefixes(n, dtype, D):
    run(plain.Shared([1, 2, 100, 1], [40, 2, 130, 500], [0, 4], [n], 4, 2, D, dtype, seed=n))


@pytest.mark.parametrize("dtype", [BF, FL])
@pytest.mark.parametrize("q_len", [[1], [31], [32], [33], [64], [65], [127], [129], [64, 64], [32, 1], [1] * 31, [1] * 33, [1] * 64, [1] * 65, [1] * 127, [1] * 130, [65, 1, 64, 66, 3], [200, 1, 300]])
def test_numbers_of_rows(dtype, q_len):
    run(plain.Shared(q_len, [n + 5 * i % 60 for i, n in enumerate(q_len)], [0, len(q_len)], [150], 2, 2, 64, dtype))


@pytest.mark.parametrize("G,q_len", [(32, [1, 1]), (33, [1, 2, 1]), (64, [1, 1, 1]), (65, [1, 1]), (100, [2, 1]), (3, [21, 22, 1])])
def test_large_and_odd_groups_of_heads(G, q_len):
    run(plain.Shared(q_len, [60] * len(q_len), [0, len(q_len)], [90], 2 * G, 2, 64, HF))


@pytest.mark.parametrize("starts,pre", [([0, 0, 3, 3, 8, 8], [10, 200, 30, 77, 5]), ([2, 5, 6], [100, 50]), ([0, 8], [0]), ([8, 8], [100]), ([0, 0], [100]), ([0, 4, 8], [0, 64]),
                                        (list(range(9)), [16 * i + 1 for i in range(8)])])
def test_groups(starts, pre):
    run(plain.Shared([1, 3, 1, 50, 1, 0, 1, 70], [20, 3, 90, 50, 7, 30, 1, 200], starts, pre, 4, 2, 64, BF, pad=1))


def test_rows_in_front_of_the_first_own_token():
    run(plain.Shared([5, 3, 90, 2, 80], [3, 0, 40, 2, 0], [0, 3], [100], 4, 2, 64, BF))
    run(plain.Shared([5, 3, 90, 2], [3, 0, 40, 0], [0, 4], [0], 4, 2, 64, HF))


def test_many_requests_and_groups():
    n = [1 + (7 * i) % 90 for i in range(200)]
    q = [0 if i % 7 == 3 else 1 if i % 3 else min(k, 20) for i, k in enumerate(n)]
    run(plain.Shared(q, n, [0, 200], [300], 4, 2, 64, BF, pad=3))
    run(plain.Shared(q, n, list(range(0, 201, 2)), [1 + (13 * g) % 150 for g in range(100)], 4, 2, 64, HF))


def test_more_requests_than_the_plan_takes_at_a_time():
    R = 1100
    run(plain.Shared([1] * R, [1 + i % 20 for i in range(R)], [3, 1050], [70], 2, 1, 64, BF))
    run(plain.Shared([1] * R, [1 + i % 20 for i in range(R)], list(range(0, 1025)), [1 + g % 40 for g in range(1024)], 2, 1, 64, BF))


def test_long_ranges_are_split():
    run(plain.Shared([1] * 40, [5 + 30 * i for i in range(40)], [0, 40], [9000], 8, 2, 128, BF, page=64))
    run(plain.Shared([1, 1, 300], [4000, 10, 300], [0, 3], [20000], 4, 2, 64, HF, page=64))
    run(plain.Shared([1, 100], [6000, 100], [1, 2], [3000], 2, 1, 64, FL, page=64))


def test_a_scale_of_the_callers_and_large_logits():
    run(plain.Shared([1, 70], [60, 80], [0, 2], [200], 4, 2, 64, BF), sm_scale=0.3)
    s = plain.Shared([1, 1, 70], [60, 200, 80], [0, 3], [200], 4, 2, 64, FL, q_scale=8.0)
    run(s)


def test_strides_of_rows():
    s = plain.Shared([1, 60, 2], [20, 90, 30], [0, 3], [100], 6, 2, 64, BF, pad=2)
    p = s.p
    want, norm = run(s)
    wide = torch.full((p.T, 3, 6, 128), math.nan, dtype=BF, device=DEV)
    wide[:, 1, :, 64:] = p.q
    q = wide[:, 1, :, 64:]
    for x in (q, q.permute(1, 0, 2)[None]):
        store = torch.full((p.T, 2, 6, 64), 7.0, dtype=BF, device=DEV)
        out = store[:, 0] if x.dim() == 3 else store[:, 0].permute(1, 0, 2)[None]
        got, lse = zb.zc_paged_shared_attention(x, *s.args()[1:], out=out)
        n = p.start[-1]
        assert torch.equal(store[:n, 0], want[:n]) and bool((store[:, 1] == 7.0).all()) and torch.equal(lse[:, :n], norm[:, :n])


def test_missing_pages_read_as_zeros():
    s = plain.Shared([1, 60, 1], [40, 90, 30], [0, 3], [100], 4, 2, 64, FL)
    for r, c, bad in ((0, 1, -1), (1, 3, 10 ** 9), (3, 2, -2 ** 31), (3, 6, 2 ** 31 - 1)):
        s.p.table[r, c] = bad
        for x in (s.p.k, s.p.v):
            x[r][:, 16 * c:16 * (c + 1)] = 0
    run(s)


def test_lengths_outside_the_tables_are_the_nearest():
    s = plain.Shared([1, 60], [48, 160], [0, 2], [96], 4, 2, 64, BF)
    want = run(s)
    s.kv, s.pre = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([48, 10 ** 9], [2 ** 31 - 1]))
    pre_table = s.pre_table[:, :6]
    got = zb.zc_paged_shared_attention(*s.args()[:3], pre_table, *s.args()[4:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    s.groups = torch.tensor([-5, 10 ** 9], dtype=torch.int32, device=DEV)
    got = zb.zc_paged_shared_attention(*s.args()[:3], pre_table, *s.args()[4:])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    s.pre = torch.tensor([-3], dtype=torch.int32, device=DEV)
    s.pre_len = [0]
    s.kv = torch.tensor([48, 160], dtype=torch.int32, device=DEV)
    s.group_start = [0, 2]
    run(s)


def test_without_prefixes_it_is_the_paged_attention():
    s = plain.Shared([1, 60, 1], [3000, 90, 30], [0], [], 4, 2, 64, BF)
    p = s.p
    want = zb.zc_paged_attention(p.q, p.kp, p.vp, s.table, s.q_start, s.kv)
    for pre_table, pre, groups in ((s.pre_table, s.pre, s.groups), (s.table[:1, :0], s.kv[:1], s.q_start[:2].contiguous())):
        got = zb.zc_paged_shared_attention(p.q, p.kp, p.vp, pre_table, pre, groups, s.table, s.q_start, s.kv)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_a_prefix_in_every_request_s_own_pages_gives_the_same():
    """The paged attention over tables that begin with the prefix's pages (of whole pages)."""
    s = plain.Shared([1, 50, 1, 2], [40, 90, 300, 2], [0, 4], [160], 4, 2, 64, FL)
    p = s.p
    out, lse = run(s)
    table = torch.cat([s.pre_table[:, :10].expand(4, 10), s.table], 1).contiguous()
    want, norm = zb.zc_paged_attention(p.q, p.kp, p.vp, table, s.q_start, s.kv + 160)
    # (both are within a few fp32 roundings of the same value, values of size 1)
    assert float((out - want).abs().max()) < 2e-5 and float((lse - norm).abs().max()) < 2e-5


def test_equal_calls_have_equal_results_and_graphs_replay():
    steps = [plain.Shared([1] * 20, [5 + 30 * i for i in range(20)], [0, 20], [3000], 8, 2, 128, BF, seed=1),
             plain.Shared([1, 100, 1, 1], [3000, 700, 64, 5], [1, 4], [500], 8, 2, 64, HF, seed=2)]
    want = [run(s) for s in steps]
    now = [[torch.zeros_like(x) for x in w] for w in want]

    def call(i):
        zb.zc_paged_shared_attention(*steps[i].args(), out=now[i][0], lse=now[i][1])
    graphs = []
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for turn in range(4):
        for i in (0, 1):
            for x in now[0] + now[1]:
                x.fill_(7.0)
            call(1 - i)
            graphs[i].replay()
            torch.cuda.synchronize()
            for w, x in zip(want, now):
                n = steps[0 if w is want[0] else 1].p.start[-1]
                assert torch.equal(w[0][:n], x[0][:n]) and torch.equal(w[1][:, :n], x[1][:, :n])


def test_a_captured_step_replays_with_other_lengths():
    a = plain.Shared([1, 60, 1, 3], [30, 60, 200, 9], [0, 3], [300], 4, 2, 64, BF, seed=3, pad=30)
    out, lse = torch.zeros_like(a.p.q), torch.zeros(4, a.p.T, dtype=torch.float32, device=DEV)
    zb.zc_paged_shared_attention(*a.args(), out=out, lse=lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zb.zc_paged_shared_attention(*a.args(), out=out, lse=lse)
    g.replay()
    a.check(out, lse)
    # fewer tokens of the prefix, other groups, other chunks: of the same pages and rows
    p = a.p
    p.q[65:70] = 0.5
    p.q_len[:4], p.kv_len[:4], p.kv_len[4] = [1, 4, 50, 8], [17, 33, 150, 8], 123
    p.start = [0, 1, 5, 55, 63, 63]
    for r in range(5):
        p.k[r], p.v[r] = p.k[r][:, :p.kv_len[r]], p.v[r][:, :p.kv_len[r]]
    a.group_start, a.pre_len = [1, 4], [123]
    a.q_start.copy_(torch.tensor(p.start[:5]))
    a.kv.copy_(torch.tensor(p.kv_len[:4]))
    a.groups.copy_(torch.tensor(a.group_start))
    a.pre.copy_(torch.tensor(a.pre_len))
    for _ in range(3):
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        a.check(out, lse)
        assert bool((out[63:] == 7.0).all())


def test_threads_that_share_a_stream_and_calls_on_two():
    steps = [plain.Shared([1] * 12, [50 + 30 * i for i in range(12)], [0, 12], [2000], 8, 2, 128, BF, seed=s) for s in (3, 4)]
    want = [run(s) for s in steps]
    torch.cuda.synchronize()
    for streams in ([torch.cuda.current_stream()] * 2, [torch.cuda.Stream(), torch.cuda.Stream()]):
        out = [None, None]

        def work(n):
            with torch.cuda.stream(streams[n]):
                out[n] = [zb.zc_paged_shared_attention(*steps[n].args()) for _ in range(20)]
            streams[n].synchronize()
        threads = [threading.Thread(target=work, args=(n,)) for n in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        for results, w in zip(out, want):
            assert all(torch.equal(x, w[0]) and torch.equal(y, w[1]) for x, y in results)


# ---- prefixes long enough, and of requests enough, that their rows go through them together -------------------------
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,by_head", [(BF, 128, 8, 2, 16, True), (HF, 64, 4, 4, 32, False), (FL, 64, 6, 2, 64, True), (FL, 128, 4, 1, 16, False),
                                                         (BF, 64, 8, 1, 128, True), (HF, 128, 3, 3, 16, True)])
def test_rows_that_go_together(dtype, D, Hq, Hkv, page, by_head):
    kw = dict(page=page, by_head=by_head, pad=2)
    run(plain.Shared([1] * 24, [1 + 13 * i for i in range(24)], [0, 24], [5000], Hq, Hkv, D, dtype, **kw))
    # with chunks that go alone, requests that have no tokens, some in front of the groups and some behind
    q = [1, 3, 0, 1, 200, 1, 2, 1, 1, 70, 1, 5, 1, 1, 0, 1, 1, 16, 1, 1, 1, 90, 1, 1]
    run(plain.Shared(q, [n + 11 * i for i, n in enumerate(q)], [2, 9, 9, 21], [4700, 100, 4001], Hq, Hkv, D, dtype, **kw))


@pytest.mark.parametrize("n", [1, 63, 64, 65, 127, 1000])
@pytest.mark.parametrize("dtype", [HF, FL])
def test_short_prefixes_beside_a_long_one(n, dtype):
    run(plain.Shared([1] * 20, [3 + 7 * i for i in range(20)], [0, 6, 20], [n, 5000], 4, 2, 64, dtype, seed=n))


@pytest.mark.parametrize("G,q_len", [(1, [1] * 31), (1, [1] * 33), (1, [64, 64] * 10), (1, [63, 1, 65, 2] * 6), (2, [1] * 64), (2, [1] * 65), (3, [21, 1, 22] * 8),
                                     (5, [1] * 26), (5, [12, 13] * 10), (7, [1, 9, 2] * 7), (33, [1] * 20), (64, [1] * 20), (65, [1] * 20)])
@pytest.mark.parametrize("dtype", [BF, FL])
def test_blocks_of_rows_that_go_together(G, q_len, dtype):
    run(plain.Shared(q_len, [n + 5 * i % 60 for i, n in enumerate(q_len)], [0, len(q_len)], [3500], 2 * G, 2, 64, dtype))


@pytest.mark.parametrize("dtype,D", [(BF, 128), (HF, 64), (FL, 64), (FL, 128)])
@pytest.mark.parametrize("R", [12, 13])
def test_blocks_of_one_length(dtype, D, R):
    run(plain.Shared([66] * R, [70 + i for i in range(R)], [0, R], [4096], 8, 8, D, dtype))


@pytest.mark.parametrize("rows,dtype", [(32, BF), (33, BF), (64, BF), (40, FL)])
def test_prefixes_that_caches_do_not_hold(rows, dtype):
    """More than 128 MB of keys and values for up to 64 rows, beside a short prefix."""
    n = 33000 if dtype == BF else 17000
    run(plain.Shared([1] * (rows + 10), [2 + 5 * i for i in range(rows + 10)], [0, rows, rows + 9], [n, 700], 16, 16, 64, dtype, page=128))


@pytest.mark.parametrize("R,Hq,Hkv,D,dtype", [(100, 8, 8, 64, BF), (100, 8, 8, 64, FL), (300, 8, 4, 128, HF), (270, 4, 4, 64, BF)])
def test_long_requests_go_first(R, Hq, Hkv, D, dtype):
    """More units than run at a time, of requests of unlike lengths, some without tokens."""
    n = [1 + (97 * i) % 600 for i in range(R)]
    run(plain.Shared([0 if i % 11 == 5 else 1 + (i % 13 == 0) for i in range(R)], n, [1, R - 2], [1000], Hq, Hkv, D, dtype))


@pytest.mark.parametrize("dtype", [BF, FL])
@pytest.mark.parametrize("q_len,pre", [([1] * 20, 4000), ([1, 2, 70], 130), ([1], 100)])
def test_logits_of_minus_infinity(dtype, q_len, pre):
    """Keys of which no row has any weight, whole tiles of a prefix and of own tokens among them: as keys of very small logits.  All keys: zeros."""
    R = len(q_len)
    s = plain.Shared(q_len, [200 + i for i in range(R)], [0, R], [pre], 4, 2, 128, dtype, page=16)
    p = s.p
    p.q[:, :, 0] = p.q[:, :, 0].abs() + 0.5
    pre_page, own_page = s.pre_table[0].long(), s.table[0].long()

    def run_with(x, every=False):
        kp = p.kp.clone()
        for pages, n in ((pre_page, pre // 16), (own_page, 8)):
            some = pages[:n] if every else pages[:min(n, 4)] if n < 8 else torch.cat([pages[:4], pages[5:n:3]])
            kp[some, :, :, 0] = x
        if every:
            kp[:, :, :, 0] = torch.where(kp[:, :, :, 0].isnan(), kp[:, :, :, 0], x)
        args = list(s.args())
        args[1] = kp
        return zb.zc_paged_shared_attention(*args)
    (out, lse), (want, want_lse) = run_with(-math.inf), run_with(-1e4)
    T = p.start[R]
    assert torch.equal(out[:T], want[:T]) and torch.equal(lse[:, :T], want_lse[:, :T]) and bool(out[:T].isfinite().all())
    out, lse = run_with(-math.inf, every=True)
    assert bool((out[:T] == 0).all()) and bool((lse[:, :T] == -math.inf).all())


def test_many_groups_that_go_together():
    R = 300
    run(plain.Shared([1] * R, [1 + i % 90 for i in range(R)], [0] + list(range(5, 291, 5)), [900 + 7 * g for g in range(58)], 4, 2, 64, BF))
    R = 1100                                                                # (planned in front)
    run(plain.Shared([1 if i % 9 else 3 for i in range(R)], [3 + i % 20 for i in range(R)], [3, 500, 1050], [700, 1300], 2, 1, 64, BF))
    run(plain.Shared([1] * R, [3 + i % 20 for i in range(R)], [1] + list(range(76, 1077, 4)), [100 + g for g in range(251)], 4, 4, 64, HF))


def test_a_planned_step_and_a_found_one_in_one_graph():
    """Two steps of different kinds behind each other, replayed: their plans and partial results do not mix."""
    steps = [plain.Shared([1] * 900, [3 + i % 50 for i in range(900)], [0, 900], [600], 4, 2, 64, BF, seed=5),
             plain.Shared([1] * 24, [1 + 13 * i for i in range(24)], [0, 24], [5000], 8, 2, 128, BF, seed=6)]
    want = [run(s) for s in steps]
    now = [[torch.zeros_like(x) for x in w] for w in want]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        for s, x in zip(steps, now):
            zb.zc_paged_shared_attention(*s.args(), out=x[0], lse=x[1])
    for _ in range(3):
        for x in now[0] + now[1]:
            x.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        for w, x in zip(want, now):
            assert torch.equal(w[0], x[0]) and torch.equal(w[1], x[1])
