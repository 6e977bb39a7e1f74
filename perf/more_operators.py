"""Operators of a paged cache under pressure, as measurable cases.

Many requests of a server begin alike (instructions, a document, one prompt answered several times), and their
generations outgrow the memory that there is for them.  The operators, over the pages of a full-precision cache:

  shared   attention of a step's new tokens where groups of requests share a prefix: the prefix lies in pages of its own, and
           is multiplied once for all rows of its group
  scores   the attention weight that every cached token has gathered, by KV head, carried on from step to step
  evict    of every request the tokens that gathered the most, the newest and the first ones stay; they move to the front
           of the request's pages in their order, and the pages that are left go back to the list of free ones

`run` computes them in elementary torch operations, or, where `own` is set, through the entry points
of `paper_2405_14256_amd.binding`.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


# ---- cases --------------------------------------------------------------------------------------

def _case(op, R, Hq, Hkv, d, dtype, **kw):
    """R requests of kv_lo to kv_hi tokens of their own, new ones counted, of which q_lo to q_hi are new; the first
    `decoding` requests have one new token.  `pad`: rows of the step's tensors behind the last request's.  `by_head`: a
    page holds its heads one after the other, or its tokens.
    shared: `groups` prefixes of pre_lo to pre_hi tokens; the last `loose` requests have none.
    scores: `window`, `sinks` of the attention; `decay` of what was gathered before.
    evict: `keep` tokens at most stay, of which the `recent` newest and `sinks` first; `together`: the same for all heads."""
    c = {"op": op, "R": R, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype, "page": 64, "kv_lo": 1, "kv_hi": 1,
         "q_lo": 1, "q_hi": 1, "decoding": 0, "pad": 0, "by_head": True, "groups": 0, "pre_lo": 1, "pre_hi": 1, "loose": 0,
         "window": 0, "sinks": 0, "decay": 1.0, "keep": 0, "recent": 0, "together": False}
    c.update(kw)
    return c


def listed():
    def named(name, *a, **kw):
        return {"name": name, **_case(*a, **kw)}

    return [
        # eight answers to one prompt, early in their generation: latency
        named("shared_answers_8", "shared", 8, 32, 8, 128, "bf16", page=16, groups=1, pre_lo=1000, pre_hi=1000, kv_lo=20, kv_hi=200),
        # a server whose requests all begin with the same long instructions, one new token each
        named("shared_decode_64", "shared", 64, 32, 8, 128, "bf16", page=16, groups=1, pre_lo=8192, pre_hi=8192, kv_lo=64, kv_hi=1024),
        # questions to one document, each a chunk, a model without grouped heads: the most rows
        named("shared_questions_12", "shared", 12, 40, 40, 128, "fp16", page=32, groups=1, pre_lo=4096, pre_hi=4096, kv_lo=100, kv_hi=500,
              q_lo=100, q_hi=500, pad=33),
        # several prefixes and requests without one, single tokens and chunks together; small heads, token-major pages
        named("shared_mixed_fp16_24", "shared", 24, 16, 4, 64, "fp16", page=32, groups=5, pre_lo=500, pre_hi=4000, loose=4, kv_lo=30, kv_hi=900,
              q_lo=10, q_hi=120, decoding=17, by_head=False, pad=9),
        # interactive generation: what one request's new token attends to, over 4k
        named("scores_llama3_8b_4k", "scores", 1, 32, 8, 128, "bf16", kv_lo=4096, kv_hi=4096),
        # batched serving: requests of all lengths, one new token each
        named("scores_ragged_64", "scores", 64, 32, 8, 128, "bf16", page=16, kv_lo=64, kv_hi=8192),
        # a chunk of a long prompt, over all of the prompt before it: the most arithmetic
        named("scores_chunk_llama3_8b_16k", "scores", 1, 32, 8, 128, "bf16", kv_lo=16384, kv_hi=16384, q_lo=2048, q_hi=2048),
        # a small fp32 model's chunks under a window, older weight fading
        named("scores_window_fp32_3", "scores", 3, 8, 8, 64, "fp32", page=16, kv_lo=300, kv_hi=1000, q_lo=60, q_hi=200, window=256, sinks=4,
              decay=0.9, pad=5),
        # a 4k prompt cut to the share that compression holds salient, each head its own tokens
        named("evict_llama3_8b_4k", "evict", 1, 32, 8, 128, "bf16", kv_lo=4096, kv_hi=4096, keep=1638, recent=200, sinks=4),
        # a server that makes room: requests of all lengths, those that fit the budget stay whole
        named("evict_ragged_32", "evict", 32, 32, 8, 128, "bf16", page=16, kv_lo=500, kv_hi=8192, keep=2048, recent=256, sinks=4),
        # a batch of long prompts without grouped heads, one choice for all heads, token-major pages: the most bytes
        named("evict_llama2_13b_4k_b16", "evict", 16, 40, 40, 128, "fp16", page=16, kv_lo=3500, kv_hi=4096, keep=1024, recent=100, by_head=False,
              together=True),
        # a small fp32 model that holds 256 tokens a request
        named("evict_small_fp32_4", "evict", 4, 8, 8, 64, "fp32", page=16, kv_lo=257, kv_hi=400, keep=256, recent=64, sinks=2),
    ]


SHAPES = ((8, 8, 64), (16, 4, 64), (12, 12, 64), (32, 8, 128), (32, 4, 128), (24, 8, 64), (16, 16, 128), (40, 40, 128), (8, 1, 128))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    costs = [work(c) for c in listed()]
    top_flops, top_bytes = max(w["flops"] for w in costs), max(w["bytes"] for w in costs)
    while True:
        op = rng.choice(("shared", "scores", "evict"))
        shape, dtype = rng.choice(SHAPES), rng.choice(("bf16", "bf16", "fp16", "fp16", "fp32"))
        kw = {"page": rng.choice((16, 16, 32, 64, 128)), "by_head": rng.random() < 0.7, "pad": rng.choice((0, 0, rng.randint(1, 99)))}
        R = _log_int(rng, 1, {"shared": 96, "scores": 64, "evict": 48}[op])
        kw["kv_hi"] = _log_int(rng, 1, {"shared": 4096, "scores": 16384, "evict": 16384}[op])
        kw["kv_lo"] = max(1, int(kw["kv_hi"] * rng.uniform(0.02, 1.0)))
        if op == "evict":
            kw["pad"] = 0
            kw["keep"] = max(1, int(kw["kv_hi"] * rng.uniform(0.05, 1.0)))
            kw["recent"] = int(kw["keep"] * rng.choice((0.0, rng.uniform(0.0, 1.0))))
            kw["sinks"], kw["together"] = rng.choice((0, 4, rng.randint(1, 40))), rng.random() < 0.4
        elif rng.random() < 0.5:
            kw["q_hi"] = min(kw["kv_hi"], _log_int(rng, 2, 2048))
            kw["q_lo"] = max(1, int(kw["q_hi"] * rng.uniform(0.2, 1.0)))
            kw["decoding"] = rng.choice((0, rng.randint(0, R - 1) if R > 1 else 0))
        if op == "shared":
            kw["groups"] = rng.randint(1, min(8, R))
            kw["pre_hi"] = _log_int(rng, 1, 16384)
            kw["pre_lo"] = max(1, int(kw["pre_hi"] * rng.uniform(0.1, 1.0)))
            kw["loose"] = rng.choice((0, 0, rng.randint(0, R - kw["groups"])))
        elif op == "scores":
            kw["decay"] = rng.choice((1.0, 1.0, 0.0, round(rng.uniform(0.5, 1.0), 3)))
            if rng.random() < 0.3:
                kw["window"], kw["sinks"] = _log_int(rng, 8, 4096), rng.choice((0, 4, rng.randint(1, 100)))
        c = _case(op, R, *shape, dtype, **kw)
        w = work(c)
        q_len, kv_len = _lengths(c)
        # (of the plain form, in 32 bits)
        logits = c["Hq"] * (R * max(q_len) * max(kv_len) + (sum(q_len) * c["pre_hi"] if op == "shared" else 0)) if op != "evict" else 0
        rows = R * c["Hkv"] * max(kv_len) * c["d"]
        # fp32 products run on pipes with a sixteenth of the 16-bit rate
        if (w["flops"] * (16 if dtype == "fp32" else 1) <= top_flops and w["bytes"] <= top_bytes and logits <= 2 ** 30 and rows <= 2 ** 30
                and sum(kv_len) <= 300000):
            return c


def _lengths(c):
    """(new tokens, tokens) of every request: the case's alone, spread over its range, the longest among them."""
    rng = random.Random("%d %d %d %d %d" % (c["R"], c["kv_lo"], c["kv_hi"], c["q_lo"], c["q_hi"]))
    kv = [c["kv_hi"]] + [min(c["kv_hi"], max(c["kv_lo"], _log_int(rng, c["kv_lo"], c["kv_hi"]))) for _ in range(c["R"] - 1)]
    rng.shuffle(kv)
    if c["op"] == "evict":
        return [0] * c["R"], kv
    q = [min(n, 1 if r < c["decoding"] else c["q_hi"] if r == c["decoding"] else rng.randint(c["q_lo"], c["q_hi"])) for r, n in enumerate(kv)]
    return q, kv


def _groups(c):
    """(first request of every group and the first without one, tokens of every prefix): groups of all sizes."""
    P, n = c["groups"], c["R"] - c["loose"]
    rng = random.Random("%d %d %d %d" % (P, n, c["pre_lo"], c["pre_hi"]))
    cuts = sorted(rng.sample(range(1, n), P - 1)) if P > 1 else []
    pre = [c["pre_hi"]] + [rng.randint(c["pre_lo"], c["pre_hi"]) for _ in range(P - 1)]
    rng.shuffle(pre)
    return [0] + cuts + [n], pre


# ---- inputs ---------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    R, Hq, Hkv, d, page, op, dt = c["R"], c["Hq"], c["Hkv"], c["d"], c["page"], c["op"], DTYPES[c["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    i32 = dict(dtype=torch.int32, device="cuda")

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    q_len, kv_len = _lengths(c)
    starts, pre = _groups(c) if op == "shared" else ([0], [])
    T, most = sum(q_len) + c["pad"], max(q_len)
    s = {"case": c, "T": T, "tokens": sum(q_len), "most_q": most, "kv_len": torch.tensor(kv_len, **i32)}
    # the pool: every page of the requests and prefixes, and some that nobody has; handed out in random order
    tables, at = [], 0
    lengths = [kv_len, pre]
    N = sum(-(-n // page) for many in lengths for n in many) + 8
    order = torch.randperm(N, generator=host).int()
    for many in lengths:
        table = torch.full((len(many), -(-max(many + [1]) // page)), -1, dtype=torch.int32)
        for r, n in enumerate(many):
            have = -(-n // page)
            table[r, :have] = order[at:at + have]
            at += have
        tables.append(table.cuda())
    s["table"], s["pre_table"] = tables
    gain = torch.ones(Hkv, d)                                            # outlier key channels
    for h in range(Hkv):
        gain[h, torch.randperm(d, generator=host)[:6]] = 15.0
    gain = gain.cuda()

    def pool(scale):
        x = torch.empty(N, Hkv, page, d, dtype=dt, device="cuda") if c["by_head"] else \
            torch.empty(N, page, Hkv, d, dtype=dt, device="cuda").transpose(1, 2)
        for i in range(0, N, 256):
            x[i:i + 256] = randn(*x[i:i + 256].shape) * scale
        return x

    s["kp"] = pool(gain[:, None, :])
    first = (s["pre_table"] if pre else s["table"])[:, 0].long()
    s["kp"][first, :, 0] += 3.0                                          # a sink at the first token
    if op != "scores":
        s["vp"] = pool(1.0)
    if op != "shared":
        # gathered weight: a few tokens have most of it, some have none at all
        x = torch.exp(2.0 * randn(N, Hkv, page))
        s["sp"] = torch.where(randn(N, Hkv, page) < -1.3, torch.zeros_like(x), x)
        s["sp"][first, :, 0] += 50.0
    if op == "evict":
        s["keep"] = torch.full((R,), c["keep"], **i32)
        s["free"] = torch.randperm(2 * N, generator=host).int().cuda()
        s["n_free"] = torch.tensor([N // 3], **i32)
        s["new_len"], s["n_freed"] = torch.zeros(R, **i32), torch.zeros(1, **i32)
        s["kept"] = torch.zeros(R, 1 if c["together"] else Hkv, c["keep"], **i32)
        return s
    s["q_start"] = torch.tensor(np.cumsum([0] + q_len).tolist(), **i32)
    s["q"] = (randn(T, Hq, d) + 0.25).to(dt)
    if op == "shared":
        s["group_start"], s["pre_len"] = torch.tensor(starts, **i32), torch.tensor(pre, **i32)
        s["starts"], s["pre"], s["rows"] = starts, pre, np.cumsum([0] + q_len).tolist()
        s["out"] = torch.zeros(T, Hq, d, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(Hq, T, dtype=torch.float32, device="cuda")
        return s
    # the rows' normalisers, as the step's attention left them
    s["lse"] = torch.zeros(Hq, T, dtype=torch.float32, device="cuda")
    t = 0
    for r in range(R):
        k = s["kp"][s["table"][r, :-(-kv_len[r] // page)].long()].transpose(0, 1).reshape(Hkv, -1, d)[:, :kv_len[r]].float().mT.contiguous()
        for j in range(0, q_len[r], 256):
            n = min(256, q_len[r] - j)
            x = s["q"][t + j:t + j + n].float().reshape(n, Hkv, -1, d).permute(1, 2, 0, 3).reshape(Hkv, -1, d)
            a = (torch.matmul(x, k) * (1.0 / math.sqrt(d))).reshape(Hq, n, -1)
            pos = torch.arange(kv_len[r] - q_len[r] + j, kv_len[r] - q_len[r] + j + n, device="cuda")[:, None]
            a = a.masked_fill(~_seen(c, pos, torch.arange(kv_len[r], device="cuda")[None]), -math.inf)
            s["lse"][:, t + j:t + j + n] = torch.logsumexp(a, -1)
        t += q_len[r]
    return s


def _seen(c, pos, key):
    seen = key <= pos
    return seen & ((key > pos - c["window"]) | (key < c["sinks"])) if c["window"] else seen


# ---- one pass ---------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        from paper_2405_14256_amd import binding as zb
        if op == "shared":
            return list(zb.zc_paged_shared_attention(s["q"], s["kp"], s["vp"], s["pre_table"], s["pre_len"], s["group_start"], s["table"],
                                                     s["q_start"], s["kv_len"], out=s["out"], lse=s["lse"]))
        if op == "scores":
            return [zb.zc_paged_scores(s["q"], s["kp"], s["table"], s["q_start"], s["kv_len"], s["lse"], s["sp"], window=c["window"],
                                       sinks=c["sinks"], decay=c["decay"])]
        new_len, kept, n_freed = zb.zc_paged_evict(s["kp"], s["vp"], s["sp"], s["table"], s["kv_len"], s["keep"], c["keep"], sinks=c["sinks"],
                                                   recent=c["recent"], together=c["together"], free_pages=s["free"], n_free=s["n_free"],
                                                   new_len=s["new_len"], kept=s["kept"], n_freed=s["n_freed"])
        return [s["kp"], s["vp"], s["sp"], new_len, kept, s["free"], n_freed]
    return {"shared": _shared, "scores": _scores, "evict": _evict}[op](s, c)


def _rows(pool, table):
    """[R, H, columns x page, ...] of a pool's pages (any page in the place of one that is missing)."""
    x = pool[table.clamp(min=0).long()].transpose(1, 2)                  # [R, H, columns, page, ...]
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _own_logits(s, c):
    """Logits [R, Hq, n, keys] of every request's new rows over its own tokens, what they see, the rows [R, n] and which of them there are."""
    q, q_start, kv_len, n = s["q"], s["q_start"].long(), s["kv_len"].long(), s["most_q"]
    R, Hq, Hkv, d = c["R"], c["Hq"], c["Hkv"], c["d"]
    j = torch.arange(n, device="cuda")[None]
    row = (q_start[:-1, None] + j).clamp(max=s["T"] - 1)
    x = q[row].float().reshape(R, n, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(R, Hkv, -1, d)
    k = _rows(s["kp"], s["table"]).float().transpose(2, 3).contiguous()
    logits = torch.matmul(x, k).reshape(R, Hq, n, -1) * (1.0 / math.sqrt(d))
    pos = (kv_len - (q_start[1:] - q_start[:-1]))[:, None] + j
    seen = _seen(c, pos[..., None], torch.arange(logits.shape[-1], device="cuda"))
    return logits, seen[:, None], row, j < (q_start[1:] - q_start[:-1])[:, None]


def _shared(s, c):
    Hq, Hkv, d, n = c["Hq"], c["Hkv"], c["d"], s["tokens"]
    logits, seen, row, there = _own_logits(s, c)
    logits = logits.masked_fill(~seen, -math.inf)
    top = logits.amax(-1).clamp(min=-1e30)
    p = torch.exp(logits - top[..., None])
    v = _rows(s["vp"], s["table"]).float()
    o = torch.matmul(p.reshape(c["R"], Hkv, -1, p.shape[-1]), v).reshape(*p.shape[:3], d)
    at = row[there]                                                      # rows in the order of the step
    m, l = (torch.zeros(n, Hq, device="cuda") for _ in range(2))
    acc = torch.zeros(n, Hq, d, device="cuda")
    m[at], l[at], acc[at] = (x.transpose(1, 2)[there] for x in (top, p.sum(-1), o))
    for g, tokens in enumerate(s["pre"]):
        lo, hi = s["rows"][s["starts"][g]], s["rows"][s["starts"][g + 1]]
        k, v = (_rows(s[x], s["pre_table"][g:g + 1])[0, :, :tokens].float() for x in ("kp", "vp"))
        x = s["q"][lo:hi].float().reshape(hi - lo, Hkv, -1, d).transpose(0, 1).reshape(Hkv, -1, d)
        a = torch.matmul(x, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
        t = a.amax(-1, keepdim=True)
        p = torch.exp(a - t)
        o = torch.matmul(p, v).reshape(Hkv, hi - lo, -1, d).transpose(0, 1).reshape(hi - lo, Hq, d)
        t, z = (y.reshape(Hkv, hi - lo, -1).transpose(0, 1).reshape(hi - lo, Hq) for y in (t, p.sum(-1)))
        both = torch.maximum(m[lo:hi], t)
        f, e = torch.exp(m[lo:hi] - both), torch.exp(t - both)
        acc[lo:hi] = acc[lo:hi] * f[..., None] + o * e[..., None]
        l[lo:hi] = l[lo:hi] * f + z * e
        m[lo:hi] = both
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    out[:n] = (acc / l[..., None].clamp(min=1e-30)).to(out.dtype)
    lse[:, :n] = (m + torch.log(l)).T
    return [out, lse]


def _slots(s, c, length):
    """Page and row [R, 1, tokens] of the tokens below `length` [R], and which of them there are."""
    i = torch.arange(s["table"].shape[1] * c["page"], device="cuda")
    page = s["table"].clamp(min=0).long().repeat_interleave(c["page"], 1)
    return page, i % c["page"], i[None] < length.long()[:, None]


def _scores(s, c):
    R, Hkv = c["R"], c["Hkv"]
    logits, seen, row, there = _own_logits(s, c)
    norm = s["lse"][:, row].transpose(0, 1)                              # [R, Hq, n]
    w = torch.where(seen & there[:, None, :, None], torch.exp(logits - norm[..., None]), torch.zeros((), device="cuda"))
    w = w.sum(2).reshape(R, Hkv, -1, w.shape[-1]).sum(2)
    q_len = (s["q_start"][1:] - s["q_start"][:-1]).long()
    page, at, real = _slots(s, c, s["kv_len"])
    r, i = real.nonzero(as_tuple=True)
    old = (i < (s["kv_len"] - q_len)[r])[:, None]
    before = s["sp"][page[r, i], :, at[i]]
    s["sp"][page[r, i], :, at[i]] = torch.where(old, before * c["decay"], torch.zeros_like(before)) + w[r, :, i]
    return [s["sp"]]


def _evict(s, c):
    R, Hkv, page = c["R"], c["Hkv"], c["page"]
    kv = s["kv_len"].long()
    pages, at, real = _slots(s, c, kv)
    new = torch.minimum(kv, s["keep"].long())
    score = _rows(s["sp"], s["table"])                                   # [R, Hkv, tokens]
    by = score.double().sum(1, keepdim=True).float() if c["together"] else score
    i = torch.arange(by.shape[-1], device="cuda")[None, None]
    recent = new.clamp(max=c["recent"])
    sinks = (new - recent).clamp(max=c["sinks"])
    by = by.masked_fill((i >= (kv - recent)[:, None, None]) | (i < sinks[:, None, None]), math.inf)
    by = by.masked_fill(~real[:, None], -math.inf)
    best = torch.sort(by, dim=-1, descending=True, stable=True)[1]       # of equal ones the first
    rank = torch.empty_like(best).scatter_(-1, best, i.expand_as(best))
    stays = (rank < new[:, None, None]) & real[:, None]
    most = min(c["keep"], stays.shape[-1])
    kept = torch.sort(torch.where(stays, i, i + 2 ** 30), dim=-1)[0][..., :most]
    mine = kept < 2 ** 30                                                # [R, heads, most]
    src = kept.clamp(max=i.shape[-1] - 1).expand(R, Hkv, most)
    moved = [x.gather(2, src[..., None].expand(R, Hkv, most, x.shape[-1]))
             for x in (_rows(s["kp"], s["table"]), _rows(s["vp"], s["table"]), score[..., None])]
    r, j = mine[:, 0].nonzero(as_tuple=True)
    to, row = pages[r, j], at[j]
    s["kp"][to, :, row] = moved[0][r, :, j]
    s["vp"][to, :, row] = moved[1][r, :, j]
    s["sp"][to, :, row] = moved[2][r, :, j, 0]
    out = s["kept"].clone()
    out[..., :most] = torch.where(mine, kept, 0).int()
    # pages behind the last one that is needed
    col = torch.arange(s["table"].shape[1], device="cuda")[None]
    gone = (col >= ((new + page - 1) // page)[:, None]) & (col < ((kv + page - 1) // page)[:, None])
    n_freed = gone.sum(dtype=torch.int32)
    nth = s["n_free"].long() + gone.flatten().long().cumsum(0) - 1
    s["free"][nth[gone.flatten()]] = s["table"][gone]
    return [s["kp"], s["vp"], s["sp"], new.int(), out, s["free"], n_freed[None]]


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    c = case
    q_len, kv_len = _lengths(c)
    e, T = 4 if c["dtype"] == "fp32" else 2, sum(q_len)
    row, page = c["Hkv"] * c["d"] * e, c["page"]
    if c["op"] == "evict":
        over = [n for n in kv_len if n > c["keep"]]
        stay, heads = c["keep"] * len(over), 1 if c["together"] else c["Hkv"]
        moved = (c["keep"] - min(c["sinks"], c["keep"] - c["recent"])) * len(over)
        pages = sum(-(-n // page) - -(-min(n, c["keep"]) // page) for n in kv_len)
        return {"bytes": 4.0 * c["Hkv"] * (sum(over) + 2 * moved) + 4.0 * moved * row + 4.0 * heads * (stay + sum(kv_len) - sum(over))
                + 4.0 * sum(kv_len) / page + 4.0 * pages, "flops": 0.0}
    pairs = rows = 0
    for q, n in zip(q_len, kv_len):
        pos = np.arange(n - q, n)
        if c["window"]:
            first = max(0, n - q - c["window"] + 1)                      # the first token that a window reaches
            pairs += int((np.minimum(pos + 1, c["window"]) + np.minimum(c["sinks"], np.maximum(0, pos + 1 - c["window"]))).sum())
            rows += n - first + min(c["sinks"], first)
        else:
            pairs += int((pos + 1).sum())
            rows += n
    if c["op"] == "scores":
        scored = rows if c["decay"] == 1.0 else sum(kv_len)
        return {"bytes": 1.0 * rows * row + 8.0 * scored * c["Hkv"] + T * c["Hq"] * (c["d"] * e + 4.0) + 4.0 * rows / page,
                "flops": 2.0 * c["d"] * c["Hq"] * pairs}
    starts, pre = _groups(c)
    for g, tokens in enumerate(pre):
        pairs += tokens * sum(q_len[starts[g]:starts[g + 1]])
        rows += tokens
    return {"bytes": 2.0 * rows * row + 2.0 * T * c["Hq"] * c["d"] * e + 4.0 * T * c["Hq"] + 4.0 * rows / page,
            "flops": 4.0 * c["d"] * c["Hq"] * pairs}


# ---- the definition, in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "evict":
        return None                                                      # (what is chosen and moved: no value is computed)
    s = prepare(case, seed)
    Hq, Hkv, page, d = c["Hq"], c["Hkv"], c["page"], c["d"]
    q_len, kv_len = _lengths(c)

    def tokens(pool, table, r, n, h):
        return pool[table[r, :-(-n // page)].long(), h].reshape(-1, d)[:n].double()

    def not_seen(nq, n):
        where = torch.arange(n - nq, n, device="cuda")[:, None]
        key = torch.arange(n, device="cuda")[None, :]
        hidden = key > where
        if c["window"]:
            hidden |= (where - key >= c["window"]) & (key >= c["sinks"])
        return hidden

    t0 = 0
    if c["op"] == "scores":
        sp = s["sp"].double()
        for r in range(c["R"]):
            n, nq = kv_len[r], q_len[r]
            hidden = not_seen(nq, n)
            ids, at = s["table"][r].long().repeat_interleave(page)[:n], torch.arange(n, device="cuda") % page
            for hk in range(Hkv):
                K = tokens(s["kp"], s["table"], r, n, hk)
                total = torch.zeros(n, dtype=torch.float64, device="cuda")
                for h in range(hk * Hq // Hkv, (hk + 1) * Hq // Hkv):
                    a = s["q"][t0:t0 + nq, h].double() @ K.T.contiguous() / math.sqrt(d)
                    total += torch.exp((a - s["lse"][h, t0:t0 + nq, None].double()).masked_fill(hidden, -math.inf)).sum(0)
                old = sp[ids, hk, at] * c["decay"]
                old[n - nq:] = 0.0
                sp[ids, hk, at] = old + total
            t0 += nq
        return [sp]
    starts, pre = _groups(c)
    out = torch.zeros(s["T"], Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(Hq, s["T"], dtype=torch.float64, device="cuda")
    for r in range(c["R"]):
        n, nq = kv_len[r], q_len[r]
        of = [g for g in range(len(pre)) if starts[g] <= r < starts[g + 1]]
        hidden = not_seen(nq, n)
        if of:
            hidden = torch.cat([torch.zeros(nq, pre[of[0]], dtype=torch.bool, device="cuda"), hidden], 1)
        for hk in range(Hkv):
            K, V = (torch.cat([tokens(s[p], s["pre_table"], g, pre[g], hk) for g in of] + [tokens(s[p], s["table"], r, n, hk)]) for p in ("kp", "vp"))
            for h in range(hk * Hq // Hkv, (hk + 1) * Hq // Hkv):
                a = (s["q"][t0:t0 + nq, h].double() @ K.T.contiguous() / math.sqrt(d)).masked_fill(hidden, -math.inf)
                lse[h, t0:t0 + nq] = torch.logsumexp(a, -1)
                out[t0:t0 + nq, h] = torch.softmax(a, -1) @ V
        t0 += nq
    return [out, lse]
