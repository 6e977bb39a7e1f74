"""Requests that share prefixes, in pages, and their attention in float64."""
import math

import torch

from tests import paged_plain


class Shared:
    """Requests of kv_len own tokens, the last q_len new, in groups that begin at group_start; prefixes of pre_len tokens.  All in the same pools."""

    def __init__(self, q_len, kv_len, group_start, pre_len, Hq, Hkv, D, dtype, device="cuda", **kw):
        R, P = len(q_len), len(pre_len)
        p = self.p = paged_plain.Pages(list(q_len) + [0] * P, list(kv_len) + list(pre_len), Hq, Hkv, D, dtype, device=device, **kw)
        self.R, self.P, self.group_start, self.pre_len = R, P, list(group_start), list(pre_len)
        i32 = dict(dtype=torch.int32, device=device)
        self.table, self.pre_table = p.table[:R], p.table[R:]
        self.q_start, self.kv = p.q_start[:R + 1].contiguous(), p.kv[:R].contiguous()
        self.groups, self.pre = torch.tensor(self.group_start, **i32), torch.tensor(self.pre_len, **i32).reshape(P)

    def group_of(self, r):
        return next((g for g in range(self.P) if self.group_start[g] <= r < self.group_start[g + 1]), None)

    def args(self):
        p = self.p
        return p.q, p.kp, p.vp, self.pre_table, self.pre, self.groups, self.table, self.q_start, self.kv

    def want(self, sm_scale=0.0):
        """(out [T', Hq, D], lse [Hq, T'], size of the terms of out, error that fp32 may bring to a weight, values' sum of sizes) in float64."""
        p, T = self.p, self.p.start[-1]
        dev = p.q.device
        out, size, total_v = (torch.zeros(T, p.Hq, p.D, dtype=torch.float64, device=dev) for _ in range(3))
        lse, eps = (torch.zeros(p.Hq, T, dtype=torch.float64, device=dev) for _ in range(2))
        scale = sm_scale or 1.0 / math.sqrt(p.D)
        for r in range(self.R):
            nq, kv, g = p.q_len[r], p.kv_len[r], self.group_of(r)
            if nq == 0:
                continue
            n = 0 if g is None else self.pre_len[g]
            own = torch.arange(kv, device=dev)[None] <= torch.arange(kv - nq, kv, device=dev)[:, None]
            seen = torch.cat([torch.ones(nq, n, dtype=torch.bool, device=dev), own], 1)
            rows = slice(p.start[r], p.start[r] + nq)
            for h in range(p.Hq):
                hk = h * p.Hkv // p.Hq
                k, v = (torch.cat(([x[self.R + g][hk]] if n else []) + [x[r][hk]]).double() for x in (p.k, p.v))
                q = p.q[rows, h].double()
                x = (q @ k.T * scale).masked_fill(~seen, -math.inf)
                top = x.amax(-1, keepdim=True) if n + kv else x.new_full((nq, 1), -math.inf)
                w = torch.exp(x - torch.where(top.isfinite(), top, torch.zeros_like(top)))
                total = w.sum(-1, keepdim=True)
                w = w / total.clamp(min=1e-300)
                out[rows, h], size[rows, h], total_v[rows, h] = w @ v, w @ v.abs(), v.abs().sum(0)
                lse[h, rows] = torch.where(total > 0, top + total.log(), -math.inf)[:, 0]
                # a logit: D products and their sum in fp32, each step by 2^-24 of the sum of sizes; the exponent's argument, of up
                # to 2^6, by 2^-24 of itself and the exponential by 2^-22; sums over the keys by 2^-24 a step
                absum = (q.abs() @ k.abs().T * scale).masked_fill(~seen, 0.0).amax(-1) if n + kv else q.new_zeros(nq)
                eps[h, rows] = (p.D + 4) * 2.0 ** -24 * absum + 2.0 ** -17 + (n + kv + 64) * 2.0 ** -24
        return out, lse, size, eps, total_v

    def check(self, out, lse, sm_scale=0.0):
        o, n, size, eps, total_v = self.want(sm_scale)
        T = self.p.start[-1]
        # a weight and the result are each rounded to the type, by half a step (fp16 weights below 2^-14 by 2^-25)
        u, low = {torch.float32: (2.0 ** -24, 0.0), torch.bfloat16: (2.0 ** -8, 0.0), torch.float16: (2.0 ** -11, 2.0 ** -25)}[out.dtype]
        e = eps.T[:, :, None]
        bound = (2 * e + u) * size + u * (o.abs() + 2 * e * size) + 1e-30
        if low:
            bound = bound + low * total_v + 2.0 ** -25
        got, gl = out[:T].double(), lse[:, :T].double()
        bad = ~((got - o).abs() <= bound)
        assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} outputs off, first at {bad.nonzero()[0].tolist()}: " \
                                    f"{got[bad][0].item()} for {o[bad][0].item()} +- {bound[bad][0].item()}"
        none = n == -math.inf
        assert bool((gl[none] == -math.inf).all()), "a row without keys"
        bad = ~((gl - n).abs() <= 2 * eps + 2.0 ** -22 * n.abs()) & ~none
        assert not bool(bad.any()), f"lse off at {bad.nonzero()[0].tolist()}: {gl[bad][0].item()} for {n[bad][0].item()}"
