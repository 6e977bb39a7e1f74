"""Operators of a paged full-precision cache, as measurable cases.

Between its prompt and its compression a request's keys and values lie, in full precision, in pages
of a pool that all requests share: requests come and go, their lengths differ and grow, and a prompt
may arrive in chunks.  The operators:

  tables   block tables and slot maps of one step from the requests' lengths and a list of free pages
  store    the step's new keys and values into their slots
  attend   attention of the step's new tokens - one a request or a chunk, any mixture - over the pages,
           with or without a sliding window and a few first tokens that stay visible
  load     the pages of some requests as [B, H, L, D] tensors, which is what compression reads

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
    """R requests of kv_lo to kv_hi tokens, new ones counted, of which q_lo to q_hi are new; the first `decoding`
    requests have one new token.  `pad`: rows of the step's tensors behind the last request's.  `by_head`: a page
    holds its heads one after the other, or its tokens."""
    c = {"op": op, "R": R, "Hq": Hq, "Hkv": Hkv, "d": d, "dtype": dtype, "page": 64, "kv_lo": 1, "kv_hi": 1,
         "q_lo": 1, "q_hi": 1, "decoding": 0, "pad": 0, "window": 0, "sinks": 0, "by_head": True}
    c.update(kw)
    return c


def listed():
    def named(name, *a, **kw):
        return {"name": name, **_case(*a, **kw)}

    return [
        # the bookkeeping in front of every decode step of a server: 64 requests, one token each
        named("tables_decode_64", "tables", 64, 32, 8, 128, "bf16", page=16, kv_lo=100, kv_hi=8192),
        # the same in front of an offline batch of whole prompts, ragged, padded to a fixed number of rows
        named("tables_prompts_256", "tables", 256, 32, 8, 128, "bf16", page=64, kv_lo=32, kv_hi=4096, q_lo=32, q_hi=4096, pad=1000),
        # one layer's new keys and values of a decode step: latency only
        named("store_decode_64", "store", 64, 32, 8, 128, "bf16", page=16, kv_lo=100, kv_hi=2000),
        # of eight prompts' chunks, a model without grouped heads, odd lengths
        named("store_chunks_8", "store", 8, 40, 40, 128, "fp16", page=32, kv_lo=700, kv_hi=4096, q_lo=700, q_hi=1500, pad=57),
        # a finished prompt, gathered for its compression
        named("load_llama3_8b_4k", "load", 1, 32, 8, 128, "bf16", kv_lo=4096, kv_hi=4096),
        # a batch of them without grouped heads, in pages whose tokens lie together: the most bytes
        named("load_llama2_13b_4k_b16", "load", 16, 40, 40, 128, "fp16", page=16, kv_lo=3500, kv_hi=4096, by_head=False),
        # interactive generation: one request, one new token over 4k
        named("decode_llama3_8b_4k", "attend", 1, 32, 8, 128, "bf16", kv_lo=4096, kv_hi=4096),
        # batched serving: requests of all lengths, one new token each
        named("decode_ragged_64", "attend", 64, 32, 8, 128, "bf16", page=16, kv_lo=64, kv_hi=8192),
        # a chunk of a long prompt, over all of the prompt before it: the most arithmetic
        named("chunk_llama3_8b_32k", "attend", 1, 32, 8, 128, "bf16", kv_lo=32768, kv_hi=32768, q_lo=2048, q_hi=2048),
        # a step in which some prompts' chunks and other requests' single tokens go together; small heads, token-major pages
        named("mixed_fp16_24", "attend", 24, 16, 4, 64, "fp16", page=32, kv_lo=200, kv_hi=4001, q_lo=250, q_hi=500, decoding=20,
              by_head=False, pad=9),
        # sliding-window decoding with four sinks, long ragged requests
        named("window_decode_16", "attend", 16, 32, 8, 128, "bf16", page=32, kv_lo=2000, kv_hi=32768, window=4096, sinks=4),
        # a small fp32 model's chunks under a window: launches and latency, no 16-bit operands
        named("window_chunk_fp32", "attend", 2, 8, 8, 64, "fp32", page=16, kv_lo=300, kv_hi=1000, q_lo=100, q_hi=256, window=256, sinks=4),
    ]


SHAPES = ((8, 8, 64), (16, 4, 64), (12, 12, 64), (32, 8, 128), (32, 4, 128), (24, 8, 64), (16, 16, 128), (40, 40, 128), (8, 1, 128))


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    by_name = {c["name"]: work(c) for c in listed()}
    top_flops, top_bytes = by_name["chunk_llama3_8b_32k"]["flops"], by_name["load_llama2_13b_4k_b16"]["bytes"]
    while True:
        op = rng.choice(("tables", "store", "load", "attend", "attend", "attend"))
        shape, dtype = rng.choice(SHAPES), rng.choice(("bf16", "bf16", "fp16", "fp16", "fp32"))
        kw = {"page": rng.choice((16, 16, 32, 64, 128)), "by_head": rng.random() < 0.7, "pad": rng.choice((0, 0, rng.randint(1, 99)))}
        R = _log_int(rng, 1, {"tables": 1024, "store": 64, "load": 16, "attend": 96}[op])
        kw["kv_hi"] = _log_int(rng, 16, 32768)
        kw["kv_lo"] = max(1, int(kw["kv_hi"] * rng.uniform(0.02, 1.0)))
        if op == "load":
            kw["pad"] = 0
        elif rng.random() < 0.5:
            kw["q_hi"] = min(kw["kv_hi"], _log_int(rng, 2, 4096))
            kw["q_lo"] = max(1, int(kw["q_hi"] * rng.uniform(0.2, 1.0)))
            kw["decoding"] = rng.choice((0, rng.randint(0, R - 1) if R > 1 else 0))
        if op == "attend" and rng.random() < 0.4:
            kw["window"], kw["sinks"] = _log_int(rng, 8, 4096), rng.choice((0, 4, 4, rng.randint(1, 100)))
        c = _case(op, R, *shape, dtype, **kw)
        w = work(c)
        logits = R * c["Hq"] * c["q_hi"] * c["kv_hi"] if op == "attend" else 0
        rows = R * c["Hkv"] * c["kv_hi"] * c["d"] * (1 if op == "attend" else 0)                     # (of the plain form, in 32 bits)
        # fp32 products run on pipes with a sixteenth of the 16-bit rate
        if (w["flops"] * (16 if dtype == "fp32" else 1) <= top_flops and w["bytes"] <= top_bytes and logits <= 32 * 2048 * 32768
                and rows <= 2 ** 30 and sum(_lengths(c)[1]) <= 400000):
            return c


def _lengths(c):
    """(new tokens, all tokens) of every request: the case's alone, spread over its range, the longest in front."""
    rng = random.Random("%d %d %d %d %d" % (c["R"], c["kv_lo"], c["kv_hi"], c["q_lo"], c["q_hi"]))
    kv = [c["kv_hi"]] + [min(c["kv_hi"], max(c["kv_lo"], _log_int(rng, c["kv_lo"], c["kv_hi"]))) for _ in range(c["R"] - 1)]
    rng.shuffle(kv)
    if c["op"] == "load":
        return [0] * c["R"], kv
    q = [min(n, 1 if r < c["decoding"] else c["q_hi"] if r == c["decoding"] else rng.randint(c["q_lo"], c["q_hi"])) for r, n in enumerate(kv)]
    return q, kv


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
    T, cols = sum(q_len) + c["pad"], -(-c["kv_hi"] // page)
    s = {"case": c, "T": T, "tokens": sum(q_len), "q_len": torch.tensor(q_len, **i32), "kv_len": torch.tensor(kv_len, **i32),
         "most_q": max(q_len)}
    # the pool: every page of the requests, and some that nobody has; handed out in random order
    have = [-(-n // page) for n in kv_len]
    N = sum(have) + 8
    order = torch.randperm(N, generator=host).int()
    table = torch.full((R, cols), -1, dtype=torch.int32)
    at = np.cumsum([0] + have)
    for r in range(R):
        table[r, :have[r]] = order[at[r]:at[r] + have[r]]
    if op == "tables":
        # pages of the tokens that were there before are in the table, the others are still free
        s["free"] = torch.randperm(2 * N, generator=host).int().cuda()
        s["n_free"] = torch.tensor([2 * N - 3], **i32)
        old = torch.tensor([-(-(n - q) // page) for n, q in zip(kv_len, q_len)])
        s["table"] = torch.where(torch.arange(cols)[None] < old[:, None], table, -1).cuda()
        return s
    gain = torch.ones(Hkv, d)                                            # outlier key channels
    for h in range(Hkv):
        gain[h, torch.randperm(d, generator=host)[:6]] = 15.0
    gain = gain.cuda()
    s["table"] = table.cuda()
    q_start = torch.zeros(R + 1, **i32)
    q_start[1:] = s["q_len"].cumsum(0)
    s["q_start"] = q_start

    def pool(scale):
        x = torch.empty(N, Hkv, page, d, dtype=dt, device="cuda") if c["by_head"] else \
            torch.empty(N, page, Hkv, d, dtype=dt, device="cuda").transpose(1, 2)
        for i in range(0, N, 256):
            x[i:i + 256] = randn(*x[i:i + 256].shape) * scale
        return x

    s["kp"], s["vp"] = pool(gain[:, None, :]), pool(1.0)
    s["kp"][s["table"][:, 0].long(), :, 0] += 3.0                        # a sink at every request's first token
    if op == "store":
        s["k"], s["v"] = (randn(T, Hkv, d) * gain).to(dt), randn(T, Hkv, d).to(dt)
        slots = torch.full((T,), -1, dtype=torch.int32)
        t = 0
        for r in range(R):
            pos = torch.arange(kv_len[r] - q_len[r], kv_len[r])
            slots[t:t + q_len[r]] = table[r, pos // page] * page + pos % page
            t += q_len[r]
        s["slots"] = slots.cuda()
    elif op == "load":
        s["ko"], s["vo"] = (torch.zeros(R, Hkv, c["kv_hi"], d, dtype=dt, device="cuda") for _ in range(2))
    else:
        s["q"] = (randn(T, Hq, d) + 0.25).to(dt)
        s["out"] = torch.zeros(T, Hq, d, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(Hq, T, dtype=torch.float32, device="cuda")
    return s


# ---- one pass ---------------------------------------------------------------------------------------

def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        from paper_2405_14256_amd import binding as zb
        if op == "tables":
            q_start, slots, taken = zb.zc_paged_tables(s["q_len"], s["kv_len"], s["table"], s["free"], c["page"], s["T"], n_free=s["n_free"])
            return [s["table"], q_start, slots, taken]
        if op == "store":
            zb.zc_paged_store(s["k"], s["v"], s["slots"], s["kp"], s["vp"])
            return [s["kp"], s["vp"]]
        if op == "load":
            return list(zb.zc_paged_load(s["kp"], s["vp"], s["table"], s["kv_len"], k_out=s["ko"], v_out=s["vo"]))
        return list(zb.zc_paged_attention(s["q"], s["kp"], s["vp"], s["table"], s["q_start"], s["kv_len"], window=c["window"],
                                          sinks=c["sinks"], out=s["out"], lse=s["lse"]))
    if op == "tables":
        return _tables(s, c["page"])
    if op == "store":
        n, slot = s["tokens"], s["slots"][:s["tokens"]].long()
        s["kp"][slot // c["page"], :, slot % c["page"]] = s["k"][:n]
        s["vp"][slot // c["page"], :, slot % c["page"]] = s["v"][:n]
        return [s["kp"], s["vp"]]
    if op == "load":
        there = (torch.arange(c["kv_hi"], device="cuda")[None] < s["kv_len"][:, None])[:, None, :, None]
        return [torch.where(there, _rows(s[p], s["table"])[:, :, :c["kv_hi"]], o) for p, o in (("kp", s["ko"]), ("vp", s["vo"]))]
    return _attend(s, c)


def _tables(s, page):
    q_len, kv_len, table = s["q_len"], s["kv_len"], s["table"]
    past = kv_len - q_len
    have = (past + page - 1) // page
    need = (kv_len + page - 1) // page - have
    taken = need.cumsum(0)
    col = torch.arange(table.shape[1], device="cuda")[None]
    nth = (taken - need)[:, None] + col - have[:, None]                 # among the pages taken
    fresh = (col >= have[:, None]) & (nth < taken[:, None])
    at = s["n_free"].long() - 1 - nth
    page_of = torch.where(at >= 0, s["free"][at.clamp(min=0, max=s["free"].numel() - 1)], -1)
    table = torch.where(fresh, page_of, table)
    q_start = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), q_len.cumsum(0).int()])
    t = torch.arange(s["T"], device="cuda", dtype=torch.int32)
    r = torch.searchsorted(q_start[1:], t, right=True).clamp(max=q_len.numel() - 1)
    pos = (past[r] + t - q_start[r]).clamp(min=0, max=table.shape[1] * page - 1)
    p = table[r, pos // page]
    slots = torch.where((t < q_start[-1]) & (p >= 0), p * page + pos % page, -1).int()
    return [table, q_start, slots, taken[-1:].int()]


def _rows(pool, table):
    """[R, H, columns x page, D] of a pool's pages (any page in the place of one that is missing)."""
    x = pool[table.clamp(min=0).long()]                                  # [R, columns, H, page, D]
    return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1, x.shape[4])


def _attend(s, c):
    q, q_start, kv_len, n = s["q"], s["q_start"].long(), s["kv_len"].long(), s["most_q"]
    R, Hq, Hkv, d = c["R"], c["Hq"], c["Hkv"], c["d"]
    G = Hq // Hkv
    j = torch.arange(n, device="cuda")[None]
    row = (q_start[:-1, None] + j).clamp(max=s["T"] - 1)                 # [R, n]
    x = q[row].float().reshape(R, n, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(R, Hkv, G * n, d)
    k = _rows(s["kp"], s["table"]).float().transpose(2, 3).contiguous()
    logits = torch.matmul(x, k).reshape(R, Hq, n, -1) * (1.0 / math.sqrt(d))
    pos = (kv_len - (q_start[1:] - q_start[:-1]))[:, None] + j           # [R, n]
    key = torch.arange(logits.shape[-1], device="cuda")
    seen = key <= pos[..., None]
    if c["window"]:
        seen = seen & ((key > pos[..., None] - c["window"]) | (key < c["sinks"]))
    logits = logits.masked_fill(~seen[:, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(logits - top)
    total = p.sum(-1, keepdim=True)
    v = _rows(s["vp"], s["table"]).float()
    o = torch.matmul(p.reshape(R, Hkv, G * n, -1), v).reshape(R, Hq, n, d) / total.clamp(min=1e-30)
    lse = (top + torch.log(total))[..., 0]
    t = torch.arange(s["tokens"], device="cuda")
    r = torch.searchsorted(q_start[1:].contiguous(), t, right=True)
    at = t - q_start[r]
    out, norm = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    out[:s["tokens"]] = o[r, :, at].to(q.dtype)
    norm[:, :s["tokens"]] = lse[r, :, at].T
    return [out, norm]


# ---- what a pass cannot do without -------------------------------------------------------------------

def work(case):
    c = case
    q_len, kv_len = _lengths(c)
    e, T = 4 if c["dtype"] == "fp32" else 2, sum(q_len)
    row = c["Hkv"] * c["d"] * e
    page = c["page"]
    if c["op"] == "tables":
        fresh = sum(-(-n // page) - -(-(n - q) // page) for n, q in zip(kv_len, q_len))
        return {"bytes": 4.0 * (3 * c["R"] + 2 * fresh + T + c["pad"]), "flops": 4.0 * (T + c["pad"])}
    if c["op"] == "store":
        return {"bytes": 4.0 * T + 4.0 * T * row, "flops": 0.0}
    if c["op"] == "load":
        return {"bytes": 4.0 * sum(kv_len) * row + 4.0 * sum(-(-n // page) for n in kv_len), "flops": 0.0}
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
    return {"bytes": 2.0 * rows * row + 2.0 * T * c["Hq"] * c["d"] * e + 4.0 * T * c["Hq"] + 4.0 * rows / page,
            "flops": 4.0 * c["d"] * c["Hq"] * pairs}


# ---- the definition, in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] != "attend":
        return None
    s = prepare(case, seed)
    out = torch.zeros(s["T"], c["Hq"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(c["Hq"], s["T"], dtype=torch.float64, device="cuda")
    q_len, kv_len = _lengths(c)
    t0 = 0
    for r in range(c["R"]):
        n, nq = kv_len[r], q_len[r]
        page_ids = s["table"][r, :-(-n // c["page"])].long()
        where = torch.arange(n - nq, n, device="cuda")[:, None]
        key = torch.arange(n, device="cuda")[None, :]
        hidden = key > where
        if c["window"]:
            hidden |= (where - key >= c["window"]) & (key >= c["sinks"])
        for hk in range(c["Hkv"]):
            K = torch.cat(list(s["kp"][page_ids, hk]), 0)[:n].double()
            V = torch.cat(list(s["vp"][page_ids, hk]), 0)[:n].double()
            for h in range(hk * c["Hq"] // c["Hkv"], (hk + 1) * c["Hq"] // c["Hkv"]):
                a = (s["q"][t0:t0 + nq, h].double() @ K.T.contiguous() / math.sqrt(c["d"])).masked_fill(hidden, -math.inf)
                lse[h, t0:t0 + nq] = torch.logsumexp(a, -1)
                out[t0:t0 + nq, h] = torch.softmax(a, -1) @ V
        t0 += nq
    return [out, lse]
