"""Paged attention at the ends of the ranges that its documentation allows."""
import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import paged_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, FL = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, FL])
def test_the_widest_window_over_rows_far_in_front_of_the_first_token(dtype):
    """A table with room for 2^31 - 2^16 tokens, a window one shorter, and 70 000 new tokens of a request that has 100: a row's
    position less the window passes 32 bits."""
    p = plain.Pages([70000], [100], 1, 1, 64, dtype, page=65536, seed=60)
    table = torch.full((1, 32767), -1, dtype=torch.int32, device=DEV)
    table[:, :1] = p.table[:, :1]
    window = 32767 * 65536 - 1
    out, lse = torch.full_like(p.q, 5.0), torch.full((1, p.T), 5.0, dtype=torch.float32, device=DEV)
    zb.zc_paged_attention(p.q, p.kp, p.vp, table, p.q_start, p.kv, window=window, sinks=4, out=out, lse=lse)
    p.check(out, lse, window=window, sinks=4)
    assert bool((out[:69900] == 0).all()) and bool((lse[:, :69900] == -float("inf")).all())


@pytest.mark.parametrize("T,H,D,dtype", [(2, 40, 128, BF), (300, 5, 64, FL), (9000, 8, 128, BF)])
def test_tokens_with_one_slot_leave_pieces_of_theirs(T, H, D, dtype):
    """Every 16 bytes of the slot's rows are one of the tokens', and nothing else is written."""
    g = torch.Generator(device=DEV).manual_seed(T)
    k, v = (torch.randn(T, H, D, generator=g, device=DEV).to(dtype) for _ in range(2))
    kp, vp = (torch.full((3, H, 16, D), 7.0, dtype=dtype, device=DEV) for _ in range(2))
    zb.zc_paged_store(k, v, torch.full((T,), 21, dtype=torch.int32, device=DEV), kp, vp)
    n = 16 // dtype.itemsize
    for pool, x in ((kp, k), (vp, v)):
        got = pool[1, :, 5].reshape(H, D // n, n)
        assert bool((x.reshape(T, H, D // n, n) == got).all(-1).any(0).all())
        pool[1, :, 5] = 7.0
        assert bool((pool == 7.0).all())


def test_pages_of_finished_requests_are_taken_again():
    """A pool that holds three requests' pages, twelve requests one after the other: every finished one's pages go back."""
    page, cols, N = 16, 5, 15
    i32 = dict(dtype=torch.int32, device=DEV)
    free, n_free = torch.arange(N, **i32), torch.tensor([N], **i32)
    table = torch.full((3, cols), -1, **i32)
    kv = [0, 0, 0]
    for step in range(200):
        r = step % 3
        if kv[r] == 80 - 7 * r:                                               # finished
            n = -(-kv[r] // page)
            free.index_copy_(0, n_free + torch.arange(n, device=DEV), table[r, :n])
            n_free += n
            kv[r] = 0
        new = [0, 0, 0]
        new[r] = min(9, 80 - 7 * r - kv[r])
        kv[r] += new[r]
        _, slots, taken = zb.zc_paged_tables(torch.tensor(new, **i32), torch.tensor(kv, **i32), table, free, page, sum(new), n_free=n_free)
        n_free -= taken
        held = [int(x) for i in range(3) for x in table[i, :-(-kv[i] // page)]]
        assert sorted(held + free[:int(n_free)].tolist()) == list(range(N))
        assert slots.tolist() == [int(table[r, p // page]) * page + p % page for p in range(kv[r] - new[r], kv[r])]
