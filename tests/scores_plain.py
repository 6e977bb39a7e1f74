"""The weight that cached tokens gather, written out plainly in float64."""
import math

import torch


def normalisers(p, window=0, sinks=0, sm_scale=0.0):
    """lse [Hq, T] of a paged_plain.Pages, rounded to fp32 (rows behind the last request: NaN)."""
    lse = torch.full((p.Hq, p.T), float("nan"), dtype=torch.float32, device=p.q.device)
    lse[:, :p.start[-1]] = p.want(window, sinks, sm_scale)[1].float()
    return lse


def seen(kv, nq, window, sinks, dev):
    pos = torch.arange(kv - nq, kv, device=dev)[:, None]
    key = torch.arange(kv, device=dev)[None]
    s = key <= pos
    return s & ((key > pos - window) | (key < sinks)) if window else s


def gathered(p, r, lse, old, window=0, sinks=0, sm_scale=0.0, decay=1.0):
    """(scores [Hkv, kv] of request r, how far fp32 may be off), old: [Hkv, kv] before."""
    nq, kv, dev = p.q_len[r], p.kv_len[r], p.q.device
    scale = sm_scale or 1.0 / math.sqrt(p.D)
    rows = slice(p.start[r], p.start[r] + nq)
    mask = seen(kv, nq, window, sinks, dev)
    out, off = (torch.zeros(p.Hkv, kv, dtype=torch.float64, device=dev) for _ in range(2))
    for h in range(p.Hq):
        hk = h * p.Hkv // p.Hq
        q, k = p.q[rows, h].double(), p.k[r][hk].double()
        x = q @ k.T * scale
        n = lse[h, rows].double()[:, None]
        w = torch.where(mask & (n > -math.inf), torch.exp(x - n), 0.0)
        # a logit: D products and their sum in fp32, each step by 2^-24 of the sum of sizes; the normaliser's and the difference's
        # change to base 2 by 2^-23 of either; the exponential by 2^-22
        size = (q.abs() @ k.abs().T * scale).masked_fill(~mask, 0.0)
        eps = (p.D + 4) * 2.0 ** -24 * size + 2.0 ** -23 * (x.abs() + 2 * n.abs().nan_to_num(posinf=0.0)) + 2.0 ** -22
        out[hk] += w.sum(0)
        off[hk] += (w * eps).nan_to_num().sum(0)
    off += (nq * p.Hq // p.Hkv + 4) * 2.0 ** -24 * out                     # sums over the rows
    keep = old.double() * decay
    keep[:, max(kv - nq, 0):] = 0.0
    off += 2.0 ** -23 * (keep.abs() + out)
    return keep + out, off + 1e-37
