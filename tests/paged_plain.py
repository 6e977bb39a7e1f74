"""The paged cache's operators written out plainly: lists and loops for the bookkeeping, float64 for the attention."""
import math

import torch


def tables(q_len, kv_len, table, free, n_free, page, T):
    """(block table, q_start, slot map, pages needed) as lists."""
    table = [list(row) for row in table]
    start, slots, taken = [0], [], 0
    for r, (q, kv) in enumerate(zip(q_len, kv_len)):
        kv = max(kv, 0)
        q = min(max(q, 0), kv)
        for c in range(-(-(kv - q) // page), -(-kv // page)):
            first = start[-1] + c * page - (kv - q)                       # the page's first token among the step's
            if c < len(table[r]) and first < T:
                table[r][c] = free[n_free - 1 - taken] if taken < n_free else -1
            taken += 1
        for pos in range(kv - q, kv):
            c = pos // page
            slots.append(table[r][c] * page + pos % page if c < len(table[r]) and table[r][c] >= 0 else -1)
        start.append(start[-1] + q)
    return table, start, (slots + [-1] * T)[:T], taken


class Pages:
    """Requests of kv_len tokens, the last q_len of them new, in pages handed out at random; whatever no token lies in is NaN."""

    def __init__(self, q_len, kv_len, Hq, Hkv, D, dtype, page=16, by_head=True, seed=0, device="cuda", pad=0, spare=3, q_scale=1.0):
        g = torch.Generator(device=device).manual_seed(seed)
        host = torch.Generator().manual_seed(seed)
        self.q_len, self.kv_len, self.Hq, self.Hkv, self.D, self.page = list(q_len), list(kv_len), Hq, Hkv, D, page
        R, have = len(self.q_len), [-(-n // page) for n in kv_len]
        N = sum(have) + spare
        order = torch.randperm(N, generator=host).int()
        cols = max(have + [1])
        table = torch.full((R, cols), -7, dtype=torch.int32)
        at = 0
        for r in range(R):
            table[r, :have[r]] = order[at:at + have[r]]
            at += have[r]
        self.table_host, self.table = table, table.to(device)
        nan = float("nan")
        shape = (N, Hkv, page, D) if by_head else (N, page, Hkv, D)
        self.kp, self.vp = (torch.full(shape, nan, dtype=dtype, device=device) for _ in range(2))
        if not by_head:
            self.kp, self.vp = self.kp.transpose(1, 2), self.vp.transpose(1, 2)
        self.k, self.v = [], []
        for r in range(R):
            k, v = (torch.randn(Hkv, kv_len[r], D, generator=g, device=device).to(dtype) for _ in range(2))
            self.k.append(k)
            self.v.append(v)
            self.write(r)
        self.T = sum(q_len) + pad
        self.q = torch.full((self.T, Hq, D), nan, dtype=dtype, device=device)
        self.q[:sum(q_len)] = (torch.randn(sum(q_len), Hq, D, generator=g, device=device) * q_scale).to(dtype)
        start = [0]
        for n in q_len:
            start.append(start[-1] + n)
        self.start = start
        i32 = dict(dtype=torch.int32, device=device)
        self.q_start, self.kv = torch.tensor(start, **i32), torch.tensor(self.kv_len, **i32)

    def write(self, r):
        """Request r's keys and values into their pages."""
        for c in range(-(-self.kv_len[r] // self.page)):
            lo, hi = c * self.page, min((c + 1) * self.page, self.kv_len[r])
            p = int(self.table_host[r, c])
            self.kp[p, :, :hi - lo] = self.k[r][:, lo:hi]
            self.vp[p, :, :hi - lo] = self.v[r][:, lo:hi]

    def want(self, window=0, sinks=0, sm_scale=0.0):
        """(out [T', Hq, D], lse [Hq, T'], size of the terms of out, error that fp32 logits and sums may bring to a weight) in float64."""
        T = self.start[-1]
        dev = self.q.device
        out, size = (torch.zeros(T, self.Hq, self.D, dtype=torch.float64, device=dev) for _ in range(2))
        lse, eps = (torch.zeros(self.Hq, T, dtype=torch.float64, device=dev) for _ in range(2))
        scale = sm_scale or 1.0 / math.sqrt(self.D)
        for r, (nq, kv) in enumerate(zip(self.q_len, self.kv_len)):
            if nq == 0:
                continue
            pos = torch.arange(kv - nq, kv, device=dev)[:, None]
            key = torch.arange(kv, device=dev)[None]
            seen = key <= pos
            if window:
                seen = seen & ((key > pos - window) | (key < sinks))
            rows = slice(self.start[r], self.start[r] + nq)
            for h in range(self.Hq):
                k, v = self.k[r][h * self.Hkv // self.Hq].double(), self.v[r][h * self.Hkv // self.Hq].double()
                q = self.q[rows, h].double()
                x = (q @ k.T * scale).masked_fill(~seen, -math.inf)
                top = x.amax(-1, keepdim=True) if kv else x.new_full((nq, 1), -math.inf)
                p = torch.exp(x - torch.where(top.isfinite(), top, torch.zeros_like(top)))
                total = p.sum(-1, keepdim=True)
                p = p / total.clamp(min=1e-300)
                out[rows, h], size[rows, h] = p @ v, p @ v.abs()
                lse[h, rows] = torch.where(total > 0, top + total.log(), -math.inf)[:, 0]
                # a logit: D products and their sum in fp32, each step by 2^-24 of the sum of sizes; the exponent's argument, of up
                # to 2^6, by 2^-24 of itself and the exponential by 2^-22; sums over the keys by 2^-24 a step
                absum = (q.abs() @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(-1) if kv else q.new_zeros(nq)
                eps[h, rows] = (self.D + 4) * 2.0 ** -24 * absum + 2.0 ** -17 + (kv + 64) * 2.0 ** -24
        return out, lse, size, eps

    def check(self, out, lse, window=0, sinks=0, sm_scale=0.0):
        """Holds out [T, Hq, D] and lse [Hq, T] against want()."""
        T = self.start[-1]
        o, n, size, eps = self.want(window, sinks, sm_scale)
        dtype = out.dtype
        # a weight and the result are each rounded to the type, by half a step (fp16 weights below 2^-14 by 2^-25)
        u, low = {torch.float32: (2.0 ** -24, 0.0), torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}[dtype]
        e = eps.T[:, :, None]
        bound = (2 * e + u) * size + u * (o.abs() + 2 * e * size) + 1e-30
        if low:
            for r, nq in enumerate(self.q_len):
                if nq and self.kv_len[r]:
                    g = self.Hq // self.Hkv
                    bound[self.start[r]:self.start[r] + nq] += low * self.v[r].double().abs().sum(1).repeat_interleave(g, 0)[None] + 2.0 ** -25
        got, gl = out[:T].double(), lse[:, :T].double()
        bad = ~((got - o).abs() <= bound)
        assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} outputs off, first at {bad.nonzero()[0].tolist()}: " \
                                    f"{got[bad][0].item()} for {o[bad][0].item()} +- {bound[bad][0].item()}"
        none = n == -math.inf
        assert bool((gl[none] == -math.inf).all()), "a row without keys"
        bad = ~((gl - n).abs() <= 2 * eps + 2.0 ** -22 * n.abs()) & ~none
        assert not bool(bad.any()), f"lse off at {bad.nonzero()[0].tolist()}: {gl[bad][0].item()} for {n[bad][0].item()}"
