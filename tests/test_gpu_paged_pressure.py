"""A server's steps as they follow each other: pages for new tokens, their keys and values, attention after a shared prefix, the weight it gathers, eviction
of what gathered least, pages that go back - against lists of rows in float64."""
import math
import random

import pytest
import torch

from paper_2405_14256_amd import binding as zb
from tests import evict_plain, shared_plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


class Server:
    def __init__(self, R, groups, pre_len, Hq, Hkv, D, dtype, page, pages, cols, seed):
        self.R, self.Hq, self.Hkv, self.D, self.dtype, self.page = R, Hq, Hkv, D, dtype, page
        self.rng, self.g = random.Random(seed), torch.Generator(device=DEV).manual_seed(seed)
        i32 = dict(dtype=torch.int32, device=DEV)
        self.kp, self.vp = (torch.full((pages, Hkv, page, D), math.nan, dtype=dtype, device=DEV) for _ in range(2))
        self.scores = torch.full((pages, Hkv, page), math.nan, device=DEV)
        self.free, self.n_free, self.pages = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int().to(DEV), torch.tensor([pages], **i32), pages
        self.table = torch.full((R, cols), -1, **i32)
        self.kv = torch.zeros(R, **i32)
        # rows of every request and head, on the host's side of the test
        self.k, self.v = ([[torch.zeros(0, D, dtype=dtype, device=DEV) for _ in range(Hkv)] for _ in range(R)] for _ in range(2))
        # the prefixes are prompts that were stored once
        P = len(pre_len)
        self.groups, self.pre_len = groups, pre_len
        self.pre_table = torch.full((max(P, 1), -(-max(pre_len + [1]) // page)), -1, **i32)
        n = torch.tensor(pre_len, **i32)
        _, slots, taken = zb.zc_paged_tables(n, n, self.pre_table, self.free, page, sum(pre_len), n_free=self.n_free)
        self.n_free -= taken
        k, v = self.rows(sum(pre_len)), self.rows(sum(pre_len))
        zb.zc_paged_store(k, v, slots, self.kp, self.vp)
        self.pre_k, self.pre_v = torch.split(k, pre_len), torch.split(v, pre_len)
        self.dgroups, self.dpre = torch.tensor(groups, **i32), n

    def rows(self, n, heads=None):
        return torch.randn(n, heads or self.Hkv, self.D, generator=self.g, device=DEV).to(self.dtype)

    def group_of(self, r):
        return next((g for g in range(len(self.pre_len)) if self.groups[g] <= r < self.groups[g + 1]), None)

    def step(self, q_len, decay):
        R, T, i32 = self.R, sum(q_len), dict(dtype=torch.int32, device=DEV)
        q, k, v = self.rows(T, self.Hq), self.rows(T), self.rows(T)
        ql = torch.tensor(q_len, **i32)
        self.kv += ql
        q_start, slots, taken = zb.zc_paged_tables(ql, self.kv, self.table, self.free, self.page, T, n_free=self.n_free)
        self.n_free -= taken
        assert int(self.n_free) >= 0
        zb.zc_paged_store(k, v, slots, self.kp, self.vp)
        old = self.scores.clone()
        out, lse = zb.zc_paged_shared_attention(q, self.kp, self.vp, self.pre_table, self.dpre, self.dgroups, self.table, q_start, self.kv)
        zb.zc_paged_scores(q, self.kp, self.table, q_start, self.kv, lse, self.scores, decay=decay)
        torch.cuda.synchronize()
        t = 0
        for r in range(R):
            for h in range(self.Hkv):
                self.k[r][h], self.v[r][h] = torch.cat([self.k[r][h], k[t:t + q_len[r], h]]), torch.cat([self.v[r][h], v[t:t + q_len[r], h]])
            self.check(r, q[t:t + q_len[r]], out[t:t + q_len[r]], lse[:, t:t + q_len[r]], old, decay)
            t += q_len[r]

    def places(self, r, n):
        i = torch.arange(n, device=DEV)
        return self.table[r].long()[i // self.page], i % self.page

    def check(self, r, q, out, lse, old, decay):
        n, nq, g = len(self.k[r][0]), len(q), self.group_of(r)
        if nq == 0:
            return
        pre = 0 if g is None else self.pre_len[g]
        seen = torch.arange(pre + n, device=DEV)[None] <= pre + torch.arange(n - nq, n, device=DEV)[:, None]
        page, row = self.places(r, n)
        # a weight and the result are each rounded to the type, by half a step (fp16 weights below 2^-14 by 2^-25)
        u, low = {FL: (2.0 ** -24, 0.0), BF: (2.0 ** -8, 0.0), HF: (2.0 ** -11, 2.0 ** -25)}[self.dtype]
        gained, off = (torch.zeros(self.Hkv, n, dtype=torch.float64, device=DEV) for _ in range(2))
        for h in range(self.Hq):
            hk = h * self.Hkv // self.Hq
            K, V = ((torch.cat([p[g][:, hk], x[r][hk]]) if pre else x[r][hk]).double() for p, x in ((self.pre_k, self.k), (self.pre_v, self.v)))
            x = (q[:, h].double() @ K.T / math.sqrt(self.D)).masked_fill(~seen, -math.inf)
            w, norm = torch.softmax(x, -1), torch.logsumexp(x, -1)
            # a logit: D products and their sum in fp32, each step by 2^-24 of the sum of sizes; the exponent's argument, of up to 2^6, by 2^-24 of
            # itself and the exponential by 2^-22; sums over the keys by 2^-24 a step
            size = (q[:, h].double().abs() @ K.abs().T / math.sqrt(self.D)).masked_fill(~seen, 0.0).amax(-1)
            eps = (self.D + 4) * 2.0 ** -24 * size + 2.0 ** -17 + (pre + n + 64) * 2.0 ** -24
            terms, want, e = w @ V.abs(), w @ V, eps[:, None]
            bound = (2 * e + u) * terms + u * (want.abs() + 2 * e * terms) + 1e-30 + low * V.abs().sum(0) + (2.0 ** -25 if low else 0.0)
            assert bool(((out[:, h].double() - want).abs() <= bound).all()), (r, h)
            assert bool(((lse[h].double() - norm).abs() <= 2 * eps + 2.0 ** -22 * norm.abs()).all()), (r, h)
            # the weights of the own tokens, by the normalisers as they came out
            a = torch.exp(x[:, pre:] - lse[h].double()[:, None])
            gained[hk] += a.sum(0)
            off[hk] += (a * (eps[:, None] + 2.0 ** -23 * (x[:, pre:].abs().nan_to_num(posinf=0.0) + 2 * lse[h].double().abs()[:, None]))).nan_to_num().sum(0)
        off += (nq * self.Hq // self.Hkv + 4) * 2.0 ** -24 * gained
        before = old[page, :, row].T.double() * decay
        before[:, n - nq:] = 0.0
        want = before + gained
        got = self.scores[page, :, row].T.double()
        assert bool(((got - want).abs() <= off + 2.0 ** -23 * want + 1e-30).all()), r

    def evict(self, keep, sinks, recent, together):
        """What stays is chosen by the scores as they are on the GPU (sums of other orders could rank two of nearly equal ones differently)."""
        R, i32 = self.R, dict(dtype=torch.int32, device=DEV)
        lists = []
        for r in range(R):
            n = len(self.k[r][0])
            page, row = self.places(r, n)
            s = self.scores[page, :, row].T.double().cpu()
            if together:
                s = s.sum(0, keepdim=True).float().double()
            lists.append([evict_plain.choose([float(x) for x in s[i]], min(n, keep[r]), sinks, recent) for i in range(len(s))])
        had = [len(self.k[r][0]) for r in range(R)]
        most = max(keep)
        new_len, kept, n_freed = zb.zc_paged_evict(self.kp, self.vp, self.scores, self.table, self.kv, torch.tensor(keep, **i32), most, sinks=sinks, recent=recent,
                                                   together=together, free_pages=self.free, n_free=self.n_free)
        self.n_free += n_freed
        self.kv = new_len
        torch.cuda.synchronize()
        for r in range(R):
            assert int(new_len[r]) == min(had[r], keep[r])
            for h in range(self.Hkv):
                at = lists[r][0 if together else h]
                assert kept[r, 0 if together else h, :len(at)].tolist() == at
                at = torch.tensor(at, dtype=torch.long, device=DEV)
                self.k[r][h], self.v[r][h] = self.k[r][h][at], self.v[r][h][at]
        L = max(int(new_len.max()), 1)
        k, v = zb.zc_paged_load(self.kp, self.vp, self.table, self.kv, L=L)
        for r in range(R):
            for h in range(self.Hkv):
                n = int(new_len[r])
                assert torch.equal(k[r, h, :n], self.k[r][h]) and torch.equal(v[r, h, :n], self.v[r][h])

    def check_pages(self):
        """Every page is free once, or in use once."""
        have = [int(x) for x in self.free[:int(self.n_free)]]
        for r in range(self.R):
            have += self.table[r, :-(-int(self.kv[r]) // self.page)].tolist()
        for g, n in enumerate(self.pre_len):
            have += self.pre_table[g, :-(-n // self.page)].tolist()
        assert sorted(have) == list(range(self.pages))


@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", [(BF, 64, 8, 2, 16), (FL, 64, 4, 4, 32), (HF, 128, 6, 2, 16)])
@pytest.mark.parametrize("together", [False, True])
def test_a_server_under_pressure(dtype, D, Hq, Hkv, page, together):
    s = Server(6, [0, 3, 5], [150, 70], Hq, Hkv, D, dtype, page, pages=60, cols=12, seed=1)
    for turn in range(6):
        s.step([s.rng.choice((1, 1, 1, 0, s.rng.randint(2, 20))) for _ in range(6)] if turn else [40, 3, 77, 20, 33, 9], decay=(1.0, 0.9)[turn % 2])
        if turn % 2:
            s.evict([20, 40, 25, 0, 64, 17], sinks=2, recent=5, together=together)
        s.check_pages()


def test_many_answers_to_a_long_prompt_under_pressure():
    """Of so many requests, after so long a prefix, that rows go through it together."""
    s = Server(40, [0, 40], [3000], 8, 2, 64, BF, 16, pages=400, cols=6, seed=2)
    for turn in range(4):
        s.step([1 + (r + turn) % 3 for r in range(40)] if turn else [1 + r % 30 for r in range(40)], decay=1.0)
        s.evict([16] * 40, sinks=0, recent=4, together=False)
        s.check_pages()


@pytest.mark.parametrize("dtype,by_head", [(BF, True), (FL, False)])
def test_offsets_past_32_bits(dtype, by_head):
    """Pools of more than 4 GB each: with the pages at their ends every operator gives what it gives with few pages."""
    s = shared_plain.Shared([1, 90, 1], [700, 333, 64], [0, 3], [500], 8, 4, 128, dtype, seed=3, page=64)
    p = s.p
    n, N = p.kp.shape[0], (5 << 30) // (4 * 64 * 128 * dtype.itemsize)
    g = torch.Generator(device=DEV).manual_seed(1)
    weights = torch.rand(n, 4, 64, generator=g, device=DEV)
    keep = torch.tensor([100, 333, 20], dtype=torch.int32, device=DEV)
    shape = (N, 4, 64, 128) if by_head else (N, 64, 4, 128)
    results = []
    for far in (False, True):
        if far:
            kp, vp = (torch.empty(shape, dtype=dtype, device=DEV) for _ in range(2))
            if not by_head:
                kp, vp = kp.transpose(1, 2), vp.transpose(1, 2)
            scores = torch.empty(N, 4, 64, device=DEV)
            kp[N - n:], vp[N - n:], scores[N - n:] = p.kp, p.vp, weights
            table, pre_table = (torch.where(t >= 0, t + N - n, t) for t in (s.table, s.pre_table))
        else:
            kp, vp, scores, table, pre_table = p.kp.clone(), p.vp.clone(), weights.clone(), s.table, s.pre_table
        out, lse = zb.zc_paged_shared_attention(p.q, kp, vp, pre_table, s.pre, s.groups, table, s.q_start, s.kv)
        zb.zc_paged_scores(p.q, kp, table, s.q_start, s.kv, lse, scores)
        new_len, kept, _ = zb.zc_paged_evict(kp, vp, scores, table, s.kv, keep, 333, sinks=2, recent=10)
        torch.cuda.synchronize()
        for r, m in enumerate((100, 333, 20)):
            kept[r, :, m:] = 0
        results.append([x.clone() for x in (out, lse, new_len, kept, kp[-n:], vp[-n:], scores[-n:])])
        s.check(out, lse)
        del kp, vp, scores
    for a, b in zip(*results):
        assert torch.equal(a.nan_to_num(-7.0) if a.is_floating_point() else a, b.nan_to_num(-7.0) if b.is_floating_point() else b)
