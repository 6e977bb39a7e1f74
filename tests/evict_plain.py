"""Eviction from a paged cache written out plainly: lists and loops, whole numbers and copies only."""
import torch


def choose(score, keep, sinks, recent):
    """The places that stay of one list of scores, ascending."""
    kv = len(score)
    stay = min(kv, max(keep, 0))
    recent = min(recent, stay)
    sinks = min(sinks, stay - recent)
    rest = sorted(range(sinks, kv - recent), key=lambda i: (-score[i], i))[:stay - recent - sinks]
    return list(range(sinks)) + sorted(rest) + list(range(kv - recent, kv))


def evict(kp, vp, sp, table, kv_len, keep, most, sinks, recent, together, kept, free, n_free):
    """Changes copies of the pools [N, Hkv, page, D], [N, Hkv, page] and lists on the CPU; returns all outputs."""
    kp, vp, sp, kept, free = (x.clone() for x in (kp, vp, sp, kept, free))
    N, H, page, _ = kp.shape
    new_len, freed = [], 0
    for r, kv in enumerate(kv_len):
        kv = min(max(kv, 0), table.shape[1] * page)
        stay = min(kv, max(keep[r], 0), most)
        new_len.append(stay)
        ids = [int(x) for x in table[r]]
        there = [0 <= p < N for p in ids]

        def score(h):
            return [float(sp[ids[i // page], h, i % page]) if there[i // page] else 0.0 for i in range(kv)]
        if together:
            rows = [score(h) for h in range(H)]
            s = [float(torch.tensor(sum(x[i] for x in rows), dtype=torch.float64).float()) for i in range(kv)]
            lists = [choose(s, stay, sinks, recent)]
        else:
            lists = [choose(score(h), stay, sinks, recent) for h in range(H)]
        for n, places in enumerate(lists):
            kept[r, n, :stay] = torch.tensor(places, dtype=torch.int32)
        for h in range(H):
            places = lists[0 if together else h]
            for x in (kp, vp, sp):
                rows = [x[ids[i // page], h, i % page].clone() if there[i // page] else torch.zeros_like(x[0, 0, 0]) for i in places]
                for to, (i, row) in enumerate(zip(places, rows)):
                    if to != i and there[to // page]:
                        x[ids[to // page], h, to % page] = row
        for c in range(-(-stay // page), -(-kv // page)):
            if 0 <= n_free + freed < len(free):
                free[n_free + freed] = ids[c]
            freed += 1
    return kp, vp, sp, torch.tensor(new_len, dtype=torch.int32), kept, free, freed
