"""The paged full-precision cache: zc_paged_tables, zc_paged_store, zc_paged_load, zc_paged_attention, and a prompt that
goes through all of them to its compression."""
import random

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from paper_2405_14256_amd import probes
from tests import paged_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32
I32 = dict(dtype=torch.int32, device=DEV)


# ---- tables ---------------------------------------------------------------------------------------------------

def _lens(rng, R, most_new, most):
    q = [rng.choice((0, 1, 1, rng.randint(0, most_new))) for _ in range(R)]
    return q, [n + rng.choice((0, rng.randint(0, most))) for n in q]


# requests, most new tokens of one, most tokens before them, page, rows behind the last, pages missing, blocks missing
TABLES = [(1, 1, 0, 16, 0, 0, 0), (1, 1, 4096, 16, 3, 0, 0), (0, 1, 1, 16, 5, 0, 0), (3, 70, 40, 16, 0, 0, 0), (64, 1, 500, 16, 0, 0, 0),
          (64, 40, 500, 64, 100, 0, 0), (65, 9, 33, 32, 1, 0, 0), (300, 3, 100, 16, 0, 5, 0), (40, 90, 90, 16, 7, 1000000, 0),
          (1023, 2, 9, 16, 0, 0, 0), (1024, 2, 9, 16, 4, 0, 0), (1025, 7, 50, 128, 0, 0, 0), (4100, 3, 70, 16, 0, 40, 1),
          (5, 9000, 3000, 16, 11, 0, 0), (30, 4000, 100, 256, 0, 0, 0), (20, 300, 100, 16, 2, 0, 3), (7, 5000, 70000, 65536, 1, 0, 0)]


@pytest.mark.parametrize("case", TABLES)
def test_tables_against_lists(case):
    R, new, before, page, pad, short, fewer = case
    rng = random.Random(repr(case))
    q_len, kv_len = _lens(rng, R, new, before)
    T = sum(q_len) + pad
    cols = max([1] + [-(-n // page) for n in kv_len]) - fewer
    table = [[rng.randint(-1, 10 ** 5) if rng.random() < 0.05 else rng.randint(0, 10 ** 5) % (0x7fffffff // page) for _ in range(cols)] for _ in range(R)]
    need = sum(-(-n // page) - -(-(n - q) // page) for q, n in zip(q_len, kv_len))
    listed = need + 4
    n_free = max(0, need - short)
    free = [rng.randint(0, min(10 ** 6, 0x7fffffff // page)) for _ in range(listed)]
    want = plain.tables(q_len, kv_len, table, free, n_free, page, T)
    wide = torch.full((R, cols + 3), -9, **I32)                              # rows with entries behind them that are nobody's
    wide[:, :cols] = torch.tensor(table, dtype=torch.int32).reshape(R, cols)
    t = wide[:, :cols]
    f = torch.tensor(free, **I32)
    start, slots, taken = zb.zc_paged_tables(torch.tensor(q_len, **I32), torch.tensor(kv_len, **I32), t, f, page, T, n_free=torch.tensor([n_free], **I32))
    assert start.tolist() == want[1] and slots.tolist() == want[2] and taken.tolist() == [want[3]] == [need]
    assert t.tolist() == want[0] and bool((wide[:, cols:] == -9).all()) and f.tolist() == free
    if n_free == need:                                                        # the whole list is free without a count
        t2 = torch.tensor(table, dtype=torch.int32).reshape(R, cols).to(DEV)
        again = zb.zc_paged_tables(torch.tensor(q_len, **I32), torch.tensor(kv_len, **I32), t2, f[:need], page, T)
        assert again[1].tolist() == slots.tolist() and t2.tolist() == want[0]


def test_tables_take_lengths_outside_their_range_for_the_nearest_and_leave_out_what_does_not_fit():
    q_len, kv_len, page = [5, -3, 40, 7], [3, 20, -1, 30], 16
    free = list(range(100, 120))
    want = plain.tables(q_len, kv_len, [[0, 1]] * 4, free, 20, page, 6)
    assert want[1] == [0, 3, 3, 3, 10]
    t = torch.tensor([[0, 1]] * 4, **I32)
    start, slots, taken = zb.zc_paged_tables(torch.tensor(q_len, **I32), torch.tensor(kv_len, **I32), t, torch.tensor(free, **I32), page, 6,
                                             n_free=torch.tensor([1000], **I32))                 # (more than the list: the list)
    assert start.tolist() == want[1] and slots.tolist() == want[2] and t.tolist() == want[0] and taken.tolist() == [want[3]]
    for n_free in (0, -5):
        t = torch.tensor([[0, 1]] * 4, **I32)
        _, slots, taken = zb.zc_paged_tables(torch.tensor(q_len, **I32), torch.tensor(kv_len, **I32), t, torch.tensor(free, **I32), page, 10,
                                             n_free=torch.tensor([n_free], **I32))
        want = plain.tables(q_len, kv_len, [[0, 1]] * 4, free, 0, page, 10)
        assert slots.tolist() == want[2] and t.tolist() == want[0] and taken.tolist() == [want[3]]


# ---- store and load -----------------------------------------------------------------------------------------------

def _pools(N, H, page, D, dtype, by_head, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if by_head:
        return [torch.randn(N, H, page, D, generator=g, device=DEV).to(dtype) for _ in range(2)]
    return [torch.randn(N, page, H, D, generator=g, device=DEV).to(dtype).transpose(1, 2) for _ in range(2)]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("case", [(1, 1, 64, 16, True), (64, 8, 128, 16, True), (65, 12, 64, 32, False), (333, 5, 128, 64, True), (2000, 40, 128, 16, False),
                                  (7, 1, 128, 16, False), (4111, 3, 64, 128, True)])
def test_store_and_load(case, dtype):
    T, H, D, page, by_head = case
    N = -(-T // page) + 9
    kp, vp = _pools(N, H, page, D, dtype, by_head, T)
    g = torch.Generator(device=DEV).manual_seed(T + 1)
    k = torch.randn(T, H, D, generator=g, device=DEV).to(dtype)
    v = torch.randn(H, T, 2 * D, generator=g, device=DEV).to(dtype)[:, :, D:].transpose(0, 1)       # another order of axes, rows apart
    slots = torch.randperm(N * page, generator=g, device=DEV)[:T].int()
    slots[::7] = torch.tensor([-1, -2 ** 31, N * page, 2 ** 31 - 1], **I32).repeat(T)[:slots[::7].numel()]     # left out
    if T > 1:
        slots[1] = N * page - 1                                               # the last slot
    slots[2:][slots[2:] == N * page - 1] = -1
    wk, wv = kp.clone(), vp.clone()
    ok = ((slots >= 0) & (slots < N * page)).nonzero()[:, 0]
    at = slots[ok].long()
    wk[at // page, :, at % page], wv[at // page, :, at % page] = k[ok], v[ok]
    zb.zc_paged_store(k, v, slots, kp, vp)
    assert torch.equal(kp, wk) and torch.equal(vp, wv)
    # and back: every page of the pool in some row of a table, entries that are no page, ragged lengths
    R, cols, L = 3, -(-N // 3) + 2, (-(-N // 3) + 2) * page - 5
    table = torch.full((R, cols + 1), -1, **I32)
    ids = torch.randperm(N, generator=g, device=DEV).int()
    for r in range(R):
        part = ids[r::R]
        table[r, :part.numel()] = part
    table[1, 0], table[2, cols - 1] = N, 2 ** 31 - 1
    kv = torch.tensor([L + 40, max(1, L // 2 + 3), 0], **I32)
    ko, vo = (torch.full((R, L, H, D), 7.0, dtype=dtype, device=DEV).transpose(1, 2) for _ in range(2))
    wide = table[:, :cols]
    got = zb.zc_paged_load(kp, vp, wide, kv, k_out=ko, v_out=vo)
    assert got[0] is ko and got[1] is vo
    for pool, o in ((kp, ko), (vp, vo)):
        rows = pool[wide.clamp(0, N - 1).long()].transpose(1, 2).reshape(R, H, cols * page, D)[:, :, :L]
        there = ((wide >= 0) & (wide < N)).repeat_interleave(page, 1)[:, :L]
        rows = torch.where(there[:, None, :, None], rows, torch.zeros_like(rows))
        inside = torch.arange(L, device=DEV)[None] < kv[:, None]
        assert torch.equal(o, torch.where(inside[:, None, :, None], rows, torch.full_like(rows, 7.0)))


def test_load_takes_no_more_tokens_than_the_table_has_room_for():
    kp, vp = _pools(5, 2, 16, 64, BF, True, 1)
    ko, vo = (torch.full((1, 2, 50, 64), 7.0, dtype=BF, device=DEV) for _ in range(2))
    zb.zc_paged_load(kp, vp, torch.tensor([[3, 4]], **I32), torch.tensor([50], **I32), k_out=ko, v_out=vo)
    assert torch.equal(ko[0, :, :32], torch.cat([kp[3], kp[4]], 1)) and bool((ko[:, :, 32:] == 7.0).all()) and bool((vo[:, :, 32:] == 7.0).all())
    k, v = zb.zc_paged_load(kp, vp, torch.tensor([[3, 4], [0, 1]], **I32), torch.tensor([32, 32], **I32))
    assert k.shape == v.shape == (2, 2, 32, 64) and torch.equal(k[1, :, :16], kp[0]) and torch.equal(v[1, :, 16:], vp[1])


# ---- attention -----------------------------------------------------------------------------------------------------

def _attend(p, window=0, sinks=0, sm_scale=0.0, out=None):
    out = torch.full_like(p.q, 5.0) if out is None else out
    lse = torch.full((p.Hq, p.T), 5.0, dtype=torch.float32, device=DEV)
    zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, window, sinks, sm_scale, out=out, lse=lse)
    n = p.start[-1]
    assert bool((out[n:] == 5.0).all()) and bool((lse[:, n:] == 5.0).all()), "rows behind the last request"
    return out, lse


def _run(q_len, kv_len, Hq, Hkv, D, dtype, window=0, sinks=0, sm_scale=0.0, **kw):
    p = plain.Pages(q_len, kv_len, Hq, Hkv, D, dtype, seed=sum(kv_len) + Hq, **kw)
    out, lse = _attend(p, window, sinks, sm_scale)
    p.check(out, lse, window, sinks, sm_scale)
    return p, out, lse


# new tokens, all tokens, query and KV heads, channels, page
SINGLE = [([1], [1], 1, 1, 64, 16), ([1], [31], 8, 8, 64, 16), ([1], [32], 8, 2, 128, 16), ([1], [33], 4, 4, 128, 32), ([1], [129], 32, 8, 128, 64),
          ([1, 1, 1], [5, 400, 63], 24, 8, 64, 16), ([1], [4097], 16, 4, 128, 128), ([1] * 70, [3 + 29 * i for i in range(70)], 8, 2, 64, 16),
          ([1] * 9, [1000 - 111 * i for i in range(9)], 40, 40, 128, 32), ([1, 1], [9000, 17], 8, 1, 128, 16), ([1], [500], 35, 5, 128, 256),
          ([1] * 130, [1 + i % 50 for i in range(130)], 4, 1, 64, 16), ([1], [700], 48, 1, 64, 16)]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("case", SINGLE)
def test_single_tokens(case, dtype):
    q, kv, Hq, Hkv, D, page = case
    _run(q, kv, Hq, Hkv, D, dtype, page=page, by_head=len(kv) % 2 == 1)


CHUNKS = [([2], [2], 2, 2, 64, 16), ([7], [40], 4, 1, 128, 16), ([33], [33], 8, 8, 64, 32), ([64], [200], 8, 2, 128, 16), ([300], [300], 4, 4, 64, 16),
          ([129], [1000], 8, 4, 128, 64), ([100, 1, 31], [100, 57, 600], 6, 2, 64, 16), ([0, 5, 0, 0, 64, 0], [9, 5, 0, 700, 65, 33], 8, 2, 128, 16),
          ([500], [1300], 12, 4, 64, 32), ([1, 1, 257, 1, 2], [300, 1, 257, 64, 900], 16, 2, 128, 16), ([1000], [1000], 3, 1, 128, 16),
          ([130, 260], [131, 261], 40, 40, 64, 128), ([17] * 66, [17 + 3 * i for i in range(66)], 4, 2, 64, 16)]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("case", CHUNKS)
def test_chunks(case, dtype):
    q, kv, Hq, Hkv, D, page = case
    _run(q, kv, Hq, Hkv, D, dtype, page=page, by_head=len(kv) % 2 == 1, pad=3)


# window, sinks
WINDOWS = [(1, 0), (1, 1), (5, 4), (16, 0), (31, 2), (64, 4), (100, 0), (100, 70), (257, 33), (1000, 4), (2 ** 31 - 1, 2 ** 31 - 1), (40, 2 ** 31 - 1)]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_windows(window, sinks, dtype):
    _run([1, 1, 1, 1], [3, 130, 700, 1500], 8, 2, 128, dtype, window=window, sinks=sinks)
    _run([60, 300, 1, 0], [60, 900, 333, 10], 4, 4, 64, dtype, window=window, sinks=sinks, page=32, by_head=False)


@pytest.mark.parametrize("dtype", [BF, HF, FL])
def test_rows_that_see_nothing(dtype):
    """A request with fewer tokens than new ones: its first rows stand in front of the first token."""
    for q, kv in (([5, 3], [2, 0]), ([1], [0]), ([200, 1], [150, 0])):
        p, out, lse = _run(q, kv, 8, 2, 64, dtype)
        assert bool((out[:q[0] - kv[0]] == 0).all()) and bool((lse[:, :q[0] - kv[0]] == -float("inf")).all())


# a request's rows in one block, in two of 32 (33 to 64 rows), in blocks of 128 (fp32: always of 32); parts of their keys joined by a second
# launch or not: new tokens, all tokens, query and KV heads, channels, page, window, sinks
BLOCKS = [([8, 9, 16, 17, 1], [8, 900, 400, 3000, 2500], 8, 2, 128, 16, 0, 0), ([33, 64, 65, 32], [33, 2000, 1100, 5000], 3, 3, 64, 32, 0, 0),
          ([512], [4000], 4, 2, 128, 64, 0, 0), ([200], [9000], 2, 1, 64, 16, 0, 0), ([130, 1, 7], [6000, 6000, 6000], 8, 4, 64, 128, 2500, 70),
          ([40, 300], [5000, 4097], 6, 1, 128, 32, 3001, 4), ([0] * 100 + [3] + [0] * 40 + [90], [50] * 100 + [2600] + [0] * 40 + [700], 8, 2, 64, 16, 0, 0),
          ([21] * 3, [4096] * 3, 12, 4, 64, 65536, 0, 0), ([1], [3000], 96, 1, 64, 16, 0, 0), ([5], [200], 70, 2, 128, 16, 50, 3)]


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("case", range(len(BLOCKS)))
def test_blocks_and_parts(case, dtype):
    q, kv, Hq, Hkv, D, page, window, sinks = BLOCKS[case]
    _run(q, kv, Hq, Hkv, D, dtype, window, sinks, page=page, by_head=case % 2 == 0, pad=case % 3)


@pytest.mark.parametrize("seed", range(40))
def test_any_lengths(seed):
    rng = random.Random(1000 + seed)
    dtype, D = rng.choice((BF, HF, FL)), rng.choice((64, 128))
    Hkv, G = rng.choice((1, 2, 3, 5)), rng.choice((1, 2, 3, 4, 7, 8, 11))
    R = rng.choice((1, 2, 5, 20, 70))
    top = 5000 // R + 40
    kv = [rng.randint(0, top) if rng.random() < 0.9 else rng.randint(0, 3) for _ in range(R)]
    q = [min(n + rng.choice((0, 0, 0, 2)), rng.choice((0, 1, 1, rng.randint(1, 20), rng.randint(1, 200)))) for n in kv]
    window, sinks = rng.choice(((0, 0), (0, 0), (rng.randint(1, 300), 0), (rng.randint(1, 2000), rng.randint(0, 99))))
    if sum(q) == 0:
        q[0], kv[0] = 1, max(kv[0], 1)
    _run(q, kv, Hkv * G, Hkv, D, dtype, window, sinks, page=rng.choice((16, 32, 64, 256)), by_head=rng.random() < 0.5, pad=rng.choice((0, 5)))


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("q,kv", [([1], [4000]), ([150], [4000])])
def test_parts_without_a_logit_above_minus_infinity(q, kv, dtype):
    """The first 2000 keys of 4000, more than one part of them, have logits of -inf: their parts weigh nothing."""
    p = plain.Pages(q, kv, 4, 2, 64, dtype, seed=4)
    p.q[..., 1] = 1.0
    p.k[0][:, :2000, 1] = -float("inf")
    p.write(0)
    out, lse = _attend(p)
    o, n, size, _ = p.want()
    u = {BF: 2.0 ** -7, HF: 2.0 ** -10, FL: 2.0 ** -13}[dtype]                 # (the weights and the result; fp32: of logits of up to 2^3)
    assert bool(((out.double() - o).abs() <= u * size + 1e-4).all()) and (lse.double() - n).abs().max().item() <= 1e-4


# (blocks of up to 32 rows over up to 2048 keys; more than 512 of them have four waves; the last: a request of many rows among empty ones)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q,kv,Hq,Hkv,window,sinks", [
    ([1], [129], 8, 8, 0, 0), ([1], [500], 32, 2, 0, 0), ([1, 0, 2, 1], [257, 90, 480, 0], 8, 2, 0, 0), ([1] * 20, [1 + 107 * i for i in range(20)], 16, 8, 0, 0),
    ([1] * 9, [1000 - 111 * i for i in range(9)], 8, 8, 0, 0), ([1] * 12, [30 * i for i in range(12)], 16, 8, 100, 5), ([1] * 5, [900, 37, 64, 300, 1], 48, 16, 130, 0),
    ([1] * 40, [25 * i + 1 for i in range(40)], 16, 8, 0, 0), ([1] * 66, [30 * i + 1 for i in range(66)], 4, 4, 0, 0), ([1] * 66, [17 * i for i in range(66)], 8, 8, 0, 0), ([0, 0, 100, 1], [10, 0, 400, 3], 4, 4, 0, 0)])
def test_blocks_of_eight_waves(q, kv, Hq, Hkv, window, sinks, D, dtype):
    _run(q, kv, Hq, Hkv, D, dtype, window, sinks, page=32, pad=2)


@pytest.mark.parametrize("q,kv,Hq,Hkv,D", [([1], [2529], 32, 4, 128), ([1, 1], [3900, 534], 12, 12, 64), ([40], [1500], 8, 2, 64)])
def test_fp32_logits_of_outlier_channels(q, kv, Hq, Hkv, D):
    """Six channels of the keys are 15 times the others: a logit's partial sums are large, and so are their roundings."""
    p = plain.Pages(q, kv, Hq, Hkv, D, FL, seed=6)
    for r in range(len(q)):
        for h in range(Hkv):
            p.k[r][h][:, torch.randperm(D, generator=torch.Generator().manual_seed(h))[:6].to(DEV)] *= 15.0
        p.write(r)
    out, lse = _attend(p)
    o, n, _, _ = p.want()
    # Relative to the result's 2-norm, the root of the summed squares, u = 2^-24, X the size of a logit (3.4 of 128 channels, 4.7 of 64): D
    # products in four sums of half the size, each addition within u / sqrt 3 of it: X sqrt(D) / 2 u / sqrt 3 = 6.6e-7 (one sum: 1.3e-6); three
    # additions u X = 2e-7; the scale's own rounding, of a few units of the exponent, 3.6e-7; the exponential 1.2e-7: 7.9e-7
    assert ((out.double() - o).norm() / o.norm()).item() < 1e-6
    assert ((lse.double() - n).norm() / n.norm()).item() < 1e-6


@pytest.mark.parametrize("dtype", [BF, HF, FL])
@pytest.mark.parametrize("q,kv", [([1], [300]), ([90], [300])])
def test_keys_whose_logits_are_minus_infinity(q, kv, dtype):
    p = plain.Pages(q, kv, 4, 2, 64, dtype, seed=3)
    p.q[..., 1] = 1.0
    for lo, hi in ((0, 40), (100, 164), (250, 251)):
        p.k[0][:, lo:hi, 1] = -float("inf")
    p.write(0)
    out, lse = _attend(p)
    o, n, size, _ = p.want()
    u = {BF: 2.0 ** -7, HF: 2.0 ** -10, FL: 2.0 ** -13}[dtype]                 # (the weights and the result; fp32: of logits of up to 2^3)
    assert bool(((out.double() - o).abs() <= u * size + 1e-4).all()) and (lse.double() - n).abs().max().item() <= 1e-4
    p.k[0][:, :, 1] = -float("inf")                                            # and of all of them
    p.write(0)
    out, lse = _attend(p)
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())


@pytest.mark.parametrize("dtype", [BF, FL])
def test_scales_strides_and_the_framework_s_order_of_axes(dtype):
    p = plain.Pages([40, 1], [90, 333], 8, 4, 64, dtype, seed=5, page=32)
    out, lse = _attend(p, sm_scale=0.3)
    p.check(out, lse, sm_scale=0.3)
    # [1, Hq, T, D], rows apart, an output with strides of its own, pools that are a slice of larger ones
    q4 = torch.zeros(1, 8, p.T, 128, dtype=dtype, device=DEV)[..., 64:]
    q4.copy_(p.q.transpose(0, 1)[None])
    kp, vp = (torch.zeros(x.shape[0], 6, x.shape[2], 192, dtype=dtype, device=DEV)[:, 1:5, :, 64:128].copy_(x) for x in (p.kp, p.vp))
    o4 = torch.zeros(1, 8, p.T, 96, dtype=dtype, device=DEV)[..., 16:80]
    table = torch.zeros(2, p.table.shape[1] + 5, **I32)
    table[:, :p.table.shape[1]] = p.table
    got = zb.zc_paged_attention(q4, kp, vp, table[:, :p.table.shape[1]], p.q_start, p.kv, sm_scale=0.3, out=o4)
    assert got[0] is o4 and torch.equal(o4[0].transpose(0, 1), out) and torch.equal(got[1], lse)
    # without outputs to write to
    o, n = zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, sm_scale=0.3)
    assert torch.equal(o, out) and torch.equal(n, lse)


@pytest.mark.parametrize("dtype", [BF, FL])
def test_pages_behind_every_window_may_be_anything(dtype):
    """Freed pages: entries that are no page, or another's page full of NaN; pages that are missing inside what is seen are zeros."""
    p = plain.Pages([1, 20], [600, 400], 8, 2, 64, dtype, seed=6)
    window, sinks = 100, 4
    nan_page = p.kp.shape[0] - 1 - int((p.table_host == p.kp.shape[0] - 1).any())
    out, lse = _attend(p, window, sinks)
    free = torch.ones(p.kp.shape[0], dtype=torch.bool)
    free[p.table_host[p.table_host >= 0].long()] = False
    nan_page = int(free.nonzero()[0])
    p.table[0, 1:30], p.table[0, 30] = -1, nan_page                            # tokens 16 .. 495 of 600; the window's first is 500
    p.table[1, 1:17] = torch.tensor([2 ** 31 - 1, nan_page], **I32).repeat(8)  # tokens 16 .. 271 of 400; 281 is the first row's first
    again = _attend(p, window, sinks)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    p.check(*again, window, sinks)
    p.table[0, 35] = -5                                                        # tokens 560 .. 575
    p.k[0][:, 560:576] = 0
    p.v[0][:, 560:576] = 0
    p.check(*_attend(p, window, sinks), window, sinks)


def test_lengths_past_the_table_are_taken_for_its_room():
    p = plain.Pages([1, 3], [64, 64], 4, 2, 64, BF, seed=7)
    out, lse = _attend(p)
    p.kv[0] = 1000
    p.kv[1] = 2 ** 31 - 1
    again = _attend(p)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_offsets_past_32_bits():
    """Pools of more than 4 GB each, with the requests' pages at their ends."""
    for dtype, by_head in ((BF, True), (FL, False)):
        small = plain.Pages([1, 90], [700, 333], 8, 4, 128, dtype, seed=8, page=64)
        N = (5 << 30) // (4 * 64 * 128 * dtype.itemsize)
        shape = (N, 4, 64, 128) if by_head else (N, 64, 4, 128)
        kp, vp = (torch.empty(shape, dtype=dtype, device=DEV) for _ in range(2))
        if not by_head:
            kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
        n = small.kp.shape[0]
        kp[N - n:], vp[N - n:] = small.kp, small.vp
        small.kp, small.vp = kp, vp
        small.table = torch.where(small.table >= 0, small.table + N - n, small.table)
        small.check(*_attend(small))
        k, v = zb.zc_paged_load(kp, vp, small.table, small.kv, L=700)
        assert torch.equal(k[0], small.k[0]) and torch.equal(v[1, :, :333], small.v[1])
        slots = torch.tensor([N * 64 - 1, (N - 1) * 64], **I32)
        zb.zc_paged_store(small.k[0][:, :2].transpose(0, 1), small.v[0][:, :2].transpose(0, 1), slots, kp, vp)
        assert torch.equal(kp[N - 1, :, 63], small.k[0][:, 0]) and torch.equal(vp[N - 1, :, 0], small.v[0][:, 1])
        del kp, vp, small


@pytest.mark.parametrize("dtype", [BF, FL])
def test_a_long_request_beside_short_ones(dtype):
    _run([1, 1, 1, 40], [30000, 20, 300, 41], 8, 2, 128, dtype, page=64)
    _run([1], [50001], 4, 4, 64, dtype, page=16)
    _run([1, 1], [20000, 20000], 8, 2, 64, dtype, page=64, window=7000, sinks=100)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_long_request_beside_a_chunk_that_fills_the_chip(dtype):
    """The chunk's blocks are whole, the long request's is in parts."""
    _run([900, 1, 1], [900, 300, 20000], 20, 20, 64, dtype, page=64)


def test_nothing_to_do():
    p = plain.Pages([1], [5], 4, 2, 64, BF)
    none = torch.zeros(0, **I32)
    out, lse = zb.zc_paged_attention(p.q[:0], p.kp, p.vp, p.table, torch.zeros(2, **I32), p.kv)
    assert out.numel() == 0 and lse.shape == (4, 0)
    out = torch.full_like(p.q, 5.0)
    zb.zc_paged_attention(p.q, p.kp, p.vp, p.table[:0], torch.zeros(1, **I32), none, out=out)
    assert bool((out == 5.0).all())
    out, lse = torch.full_like(p.q, 5.0), torch.full((4, 1), 5.0, dtype=torch.float32, device=DEV)
    zb.zc_paged_attention(p.q, p.kp, p.vp, p.table[:, :0], p.q_start, p.kv, out=out, lse=lse)          # a table without room: no token is seen
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all())
    zb.zc_paged_store(p.q[:0, :2], p.q[:0, :2], none, p.kp, p.vp)
    k, v = zb.zc_paged_load(p.kp, p.vp, p.table[:0], none)
    assert k.shape == (0, 2, 16, 64)


def test_equal_calls_give_equal_bits_on_any_stream():
    p = plain.Pages([1] * 20 + [50], [100 + 90 * i for i in range(20)] + [900], 32, 8, 128, BF, seed=9)
    out, lse = _attend(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            o2, l2 = _attend(p)
            assert torch.equal(o2, out) and torch.equal(l2, lse)
    torch.cuda.current_stream().wait_stream(side)


def test_a_captured_step_replays_with_other_lengths():
    """Tables, store and attention of a decode step in one graph, whose lengths advance on the device."""
    Hq, Hkv, D, page, dtype = 8, 2, 64, 16, BF
    R, steps, first = 5, 40, [1, 15, 16, 100, 7]
    p = plain.Pages([0] * R, first, Hq, Hkv, D, dtype, page=page, spare=60, seed=10)
    g = torch.Generator(device=DEV).manual_seed(11)
    new = [[torch.randn(R, n, D, generator=g, device=DEV).to(dtype) for n in (Hq, Hkv, Hkv)] for _ in range(steps)]
    table = torch.full((R, 12), -1, **I32)
    table[:, :p.table.shape[1]] = p.table.clamp(min=-1)
    used = set(p.table_host[p.table_host >= 0].tolist())
    spare = [i for i in range(p.kp.shape[0]) if i not in used]
    free, n_free = torch.tensor(spare, **I32), torch.tensor([len(spare)], **I32)
    ones, kv = torch.ones(R, **I32), torch.tensor(first, **I32)
    q, k, v = (torch.zeros_like(x) for x in new[0])
    out, lse = torch.zeros_like(q), torch.zeros(Hq, R, dtype=torch.float32, device=DEV)

    def step():
        kv.add_(ones)
        start, slots, taken = zb.zc_paged_tables(ones, kv, table, free, page, R, n_free=n_free)
        n_free.sub_(taken)
        zb.zc_paged_store(k, v, slots, p.kp, p.vp)
        zb.zc_paged_attention(q, p.kp, p.vp, table, start, kv, out=out, lse=lse)

    state = [x.clone() for x in (kv, table, n_free)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                                               # (scratch memory is there before the capture)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for x, s in zip((kv, table, n_free), state):
        x.copy_(s)
    for i in range(steps):
        for x, y in zip((q, k, v), new[i]):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        for r in range(R):
            p.k[r], p.v[r] = torch.cat([p.k[r], new[i][1][r][:, None]], 1), torch.cat([p.v[r], new[i][2][r][:, None]], 1)
            p.kv_len[r] += 1
        p.q_len, p.start, p.q, p.T = [1] * R, list(range(R + 1)), new[i][0], R
        if i % 7 == 0 or i == steps - 1:
            p.check(out, lse)
            eager = zb.zc_paged_attention(q, p.kp, p.vp, table, torch.arange(R + 1, **I32), kv)
            assert torch.equal(eager[0], out) and torch.equal(eager[1], lse)
    assert kv.tolist() == [n + steps for n in first]
    assert int(n_free) == len(spare) - sum(-(-(n + steps) // page) - -(-n // page) for n in first)


def test_graphs_captured_on_one_stream_replay_side_by_side():
    """Two graphs whose calls are split and joined through workspaces: each has its own."""
    ps = [plain.Pages([1, 1], [6000, 300], 8, 2, 128, BF, seed=20 + i) for i in range(2)]
    want = [_attend(p) for p in ps]
    side = torch.cuda.Stream()
    graphs, outs = [], []
    for p in ps:
        o, n = torch.zeros_like(p.q), torch.zeros(8, p.T, dtype=torch.float32, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for _ in range(20):
                zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=o, lse=n)
        graphs.append(g)
        outs.append((o, n))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    for _ in range(5):
        for (o, n) in outs:
            o.zero_()
            n.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for (o, n), (wo, wn) in zip(outs, want):
            assert torch.equal(o, wo) and torch.equal(n, wn)


def test_calls_on_two_streams_at_once():
    """Eager calls that are split and joined, on two streams without a wait between them: each stream has its own workspace."""
    ps = [plain.Pages([1, 1, 30], [5000 + 900 * i, 40, 333], 8, 2, 128, HF, seed=30 + i) for i in range(2)]
    want = [_attend(p) for p in ps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ps]
    outs = [[(torch.zeros_like(p.q), torch.zeros(8, p.T, dtype=torch.float32, device=DEV)) for _ in range(20)] for p in ps]
    torch.cuda.synchronize()
    for i in range(20):
        for p, s, o in zip(ps, streams, outs):
            with torch.cuda.stream(s):
                zb.zc_paged_attention(p.q, p.kp, p.vp, p.table, p.q_start, p.kv, out=o[i][0], lse=o[i][1])
    torch.cuda.synchronize()
    for (wo, wn), o in zip(want, outs):
        assert all(torch.equal(x, wo) and torch.equal(y, wn) for x, y in o)


def test_the_binding_refuses_what_does_not_fit():
    p = plain.Pages([1, 2], [20, 30], 4, 2, 64, BF)
    ok = (p.q, p.kp, p.vp, p.table, p.q_start, p.kv)

    def attend(error, at, value, **kw):
        args = list(ok)
        args[at] = value
        with pytest.raises(error):
            zb.zc_paged_attention(*args, **kw)
    attend(ValueError, 3, p.table.long())
    attend(ValueError, 3, p.table.cpu())
    attend(ValueError, 3, p.table[0])
    attend(ValueError, 3, p.table.T.contiguous().T)
    attend(ValueError, 3, p.table[:1].expand(2, -1))
    attend(ValueError, 4, p.q_start.long())
    attend(ValueError, 4, p.q_start[:2])
    attend(ValueError, 5, p.kv.float())
    attend(ValueError, 5, torch.cat([p.kv, p.kv]))
    attend(ValueError, 5, torch.stack([p.kv, p.kv], 1)[:, 0])
    attend(ValueError, 0, p.q.cpu())
    attend(ValueError, 0, p.q, lse=torch.zeros(4, p.T, device=DEV, dtype=torch.float64))
    attend(ValueError, 0, p.q, lse=torch.zeros(4, p.T + 1, device=DEV))
    attend(zb.ZipCacheError, 0, p.q.half())
    attend(zb.ZipCacheError, 0, p.q[:, :3])
    attend(zb.ZipCacheError, 0, p.q, out=torch.zeros(p.T, 4, 64, device=DEV))
    attend(zb.ZipCacheError, 0, p.q, window=-1)
    attend(zb.ZipCacheError, 0, p.q, sm_scale=-1.0)
    attend(AssertionError, 0, p.q[0])
    attend(AssertionError, 1, p.kp[..., ::2])
    with pytest.raises(zb.ZipCacheError):
        zb.zc_paged_attention(p.q, p.kp[:, :, :8], p.vp[:, :, :8], p.table, p.q_start, p.kv)
    slots = torch.zeros(3, **I32)
    for s in (slots.long(), slots[:2], slots.cpu()):
        with pytest.raises(ValueError):
            zb.zc_paged_store(p.q[:, :2], p.q[:, :2], s, p.kp, p.vp)
    with pytest.raises(ValueError):
        zb.zc_paged_load(p.kp, p.vp, p.table, p.kv, k_out=torch.zeros(3, 2, 8, 64, dtype=BF, device=DEV), v_out=torch.zeros(3, 2, 8, 64, dtype=BF, device=DEV))
    with pytest.raises(zb.ZipCacheError):
        zb.zc_paged_load(p.kp, p.vp, p.table, p.kv, k_out=torch.zeros(2, 2, 8, 64, dtype=BF, device=DEV), v_out=torch.zeros(2, 2, 9, 64, dtype=BF, device=DEV))
    one = torch.ones(2, **I32)
    for kw in (dict(page=12), dict(page=8)):
        with pytest.raises(zb.ZipCacheError):
            zb.zc_paged_tables(one, one, p.table, one, T=2, **kw)
    for kw in (dict(T=-1), dict(T=3, slot_map=one), dict(T=2, n_free=one), dict(T=2, q_start=one)):
        with pytest.raises(ValueError):
            zb.zc_paged_tables(one, one, p.table, one, page=16, **kw)
    torch.cuda.synchronize()


# ---- together -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, FL])
def test_prompts_in_chunks_through_the_pages_to_their_compression(dtype):
    """Two prompts arrive in chunks of different sizes, are attended over the pages, gathered, scored with the normalisers of
    their rows, split, packed and decoded: as the whole prompts are."""
    B, Hq, Hkv, D, L, page = 2, 8, 2, 128, 500, 32
    g = torch.Generator(device=DEV).manual_seed(12)
    Q, K, V = (torch.randn(B, h, L, D, generator=g, device=DEV).to(dtype) for h in (Hq, Hkv, Hkv))
    N = 2 * -(-L // page) + 4
    kp, vp = (torch.full((N, Hkv, page, D), float("nan"), dtype=dtype, device=DEV) for _ in range(2))
    table = torch.full((B, -(-L // page)), -1, **I32)
    free, n_free = torch.randperm(N, generator=g, device=DEV).int(), torch.tensor([N], **I32)
    out, lse = torch.zeros_like(Q), torch.zeros(B, Hq, L, dtype=torch.float32, device=DEV)
    done = [0, 0]
    for n in ((100, 1), (157, 300), (1, 0), (200, 199), (42, 0)):
        n = [min(x, L - d) for x, d in zip(n, done)]
        q_len, kv = torch.tensor(n, **I32), torch.tensor([d + x for d, x in zip(done, n)], **I32)
        rows = [torch.cat([x[b, :, done[b]:done[b] + n[b]].transpose(0, 1) for b in range(B)]) for x in (Q, K, V)]
        start, slots, taken = zb.zc_paged_tables(q_len, kv, table, free, page, sum(n), n_free=n_free)
        n_free -= taken
        zb.zc_paged_store(rows[1], rows[2], slots, kp, vp)
        o, s = zb.zc_paged_attention(rows[0], kp, vp, table, start, kv)
        at = 0
        for b in range(B):
            out[b, :, done[b]:done[b] + n[b]] = o[at:at + n[b]].transpose(0, 1)
            lse[b, :, done[b]:done[b] + n[b]] = s[:, at:at + n[b]]
            at += n[b]
            done[b] += n[b]
    assert done == [L, L] and int(n_free) == N - 2 * -(-L // page)
    whole, norm, _ = zb.zc_prefill_attention(Q, K, V)
    u = 2.0 ** -20 if dtype == FL else 2.0 ** -6                               # (two roundings of each, of values of up to 2^2; fp32 sums)
    assert (out.float() - whole.float()).abs().max().item() <= 4 * u and (lse - norm).abs().max().item() <= 1e-4
    k, v = zb.zc_paged_load(kp, vp, table, torch.tensor([L, L], **I32), L=L)
    assert torch.equal(k, K) and torch.equal(v, V)
    pos = torch.from_numpy(probes.probe_positions(L, 0.10, seed=0)).to(DEV)
    scores = zb.zc_probe_saliency(Q, k, pos, lse_ext=lse[:, :, pos.long()].contiguous())
    plainly = zb.zc_probe_saliency(Q, K, pos, lse_ext=norm[:, :, pos.long()].contiguous())
    # a normaliser is off by 1e-4 at most and a probability by as much of itself
    assert bool(((scores - plainly).abs() <= 2e-4 * plainly + 1e-7).all())
    salient, regular = zb.zc_select_salient(scores, 200)
    slots = zb.load().zc_arena_slots
    packed = []
    for x, y in ((k, v), (K, V)):
        Kp = zb.PackedTensor(B, Hkv, D, slots(200, 1), slots(L - 200, 1), 4, 2, "channel", zb.ZC_LAYOUT_ROW, max_chunks=1)
        Vp = zb.PackedTensor(B, Hkv, D, slots(200, 1), slots(L - 200, 1), 4, 2, "cst", zb.ZC_LAYOUT_TGROUP, max_chunks=1)
        zb.zc_quantize_pack_kv(x, y, salient, regular, Kp, Vp)
        packed.append(zb.zc_decode_attention(Q[:, :, -1], Kp, Vp))
    assert torch.equal(*packed)
