"""Cases of attention with a sliding window and sinks, of attention over a shared prefix, and of the slot maps that go with
them: what a pass through each computes, and its plain form.

A query at position i sees the positions j <= i with j < sink (the first tokens stay visible) or j > i - window.  Caches are
[B][H_kv][S_cap][W], and position p of a sequence lies in row
    p                                          if p < sink
    sink + (p - sink) mod (S_cap - sink)       else
so a cache that is long enough holds position p in row p, and a shorter one is a rolling cache whose rows behind the sinks are
used again and again.

Operators, by the key "op" of a case:
    decode   rap_decode_attn_window: the newest token of every sequence
    prefill  rap_prefill_attn_window: a block of new tokens of every sequence, as many as each has (rows of one after the other)
    shared   rap_decode_attn_shared: the newest token of every sequence; the sequences of a group share a prefix, each has its own
             rows behind it
    slots    rap_build_slots: for every new token its sequence, position and cache row, from the lengths
"""
import math

import numpy as np
import torch

own = False

HEAD_DIM = 128
# retained pairs and V channels of a head at the retain ratios 0.9, 0.8, 0.7, 0.5 and unpruned
WIDTHS = [(58, 115), (51, 102), (45, 90), (32, 64), (64, 128)]


def listed():
    return [
        # one long conversation on a rolling cache: a launch's latency
        {"name": "decode-single-4k", "op": "decode", "batch": 1, "kv_heads": 8, "group": 4, "pairs": 45, "vch": 90, "dtype": "bf16",
         "sink": 4, "window": 4096, "seq": 30011, "lens": "full", "cap": "ring"},
        # the 8B-shaped serving batch at 32K, of which a window of 4096 is kept
        {"name": "decode-batch32-4k", "op": "decode", "batch": 32, "kv_heads": 8, "group": 4, "pairs": 45, "vch": 90, "dtype": "bf16",
         "sink": 4, "window": 4096, "seq": 32769, "lens": "stairs", "cap": "ring"},
        # sequences of every length up to 9000 on a whole cache, an empty and a one-token one among them, odd V width, no sinks
        {"name": "decode-mixed-odd", "op": "decode", "batch": 24, "kv_heads": 8, "group": 3, "pairs": 58, "vch": 115, "dtype": "bf16",
         "sink": 0, "window": 1000, "seq": 9000, "lens": "mixed", "cap": "linear"},
        # a small fp32 stack
        {"name": "decode-f32-256", "op": "decode", "batch": 8, "kv_heads": 2, "group": 2, "pairs": 24, "vch": 48, "dtype": "f32",
         "sink": 4, "window": 256, "seq": 700, "lens": "stairs", "cap": "ring"},
        # a whole prompt
        {"name": "prefill-prompt-8k", "op": "prefill", "batch": 1, "kv_heads": 8, "group": 4, "pairs": 45, "vch": 90, "dtype": "bf16",
         "sink": 4, "window": 2048, "new": 8192, "news": "full", "past": 0, "lens": "full", "cap": "linear", "pad": 0},
        # chunks of long prompts on rolling caches
        {"name": "prefill-chunks-4x512", "op": "prefill", "batch": 4, "kv_heads": 8, "group": 4, "pairs": 45, "vch": 90, "dtype": "bf16",
         "sink": 4, "window": 1024, "new": 512, "news": "full", "past": 7001, "lens": "stairs", "cap": "ring", "pad": 0},
        # a step of mixed requests: chunks of every size, single tokens and idle sequences, padded to a fixed row count, odd V width
        {"name": "prefill-ragged-odd", "op": "prefill", "batch": 12, "kv_heads": 8, "group": 3, "pairs": 58, "vch": 115, "dtype": "bf16",
         "sink": 1, "window": 500, "new": 700, "news": "mixed", "past": 2500, "lens": "mixed", "cap": "ring", "pad": 37},
        # 32 answers to one prompt of 8K
        {"name": "shared-32-8k", "op": "shared", "batch": 32, "groups": 1, "kv_heads": 8, "group": 4, "pairs": 45, "vch": 90, "dtype": "bf16",
         "prefix": 8192, "prefixes": "full", "seq": 400, "lens": "mixed"},
        # 64 conversations behind one document of 32K
        {"name": "shared-64-32k", "op": "shared", "batch": 64, "groups": 1, "kv_heads": 8, "group": 4, "pairs": 45, "vch": 90, "dtype": "bf16",
         "prefix": 32769, "prefixes": "full", "seq": 1000, "lens": "stairs"},
        # several prompts of unlike lengths with a few answers each, some not begun; five query heads a KV head, odd V width
        {"name": "shared-groups-odd", "op": "shared", "batch": 23, "groups": 5, "kv_heads": 8, "group": 5, "pairs": 58, "vch": 115, "dtype": "bf16",
         "prefix": 6001, "prefixes": "mixed", "seq": 300, "lens": "mixed"},
        # the new tokens of a decode batch on rolling caches
        {"name": "slots-decode-32", "op": "slots", "batch": 32, "sink": 4, "cap_rows": 4352, "seq": 32769, "new": 1, "news": "full", "pad": 0},
        # a step of mixed requests, padded to a fixed row count
        {"name": "slots-ragged-64", "op": "slots", "batch": 64, "sink": 4, "cap_rows": 8192, "seq": 20000, "new": 900, "news": "mixed", "pad": 100},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["decode", "decode", "prefill", "prefill", "shared", "shared", "slots"])
    if op == "slots":
        return {"op": op, "batch": log(1, 500), "sink": rng.choice([0, 1, 4, 17]), "cap_rows": 8 * log(600, 4000), "seq": log(1, 100000),
                "new": log(1, 2000), "news": rng.choice(["full", "mixed"]), "pad": rng.choice([0, 0, log(1, 200)])}
    if rng.random() < 0.5:
        pairs, vch = rng.choice(WIDTHS)
    else:      # a layer-adaptive budget: V keeps twice the pairs
        pairs = rng.randint(16, 64)
        vch = 2 * pairs
    case = {"op": op, "kv_heads": rng.choice([1, 2, 4, 8]), "group": rng.randint(1, 8), "pairs": pairs, "vch": vch, "dtype": "bf16"}
    heads = case["kv_heads"] * case["group"]
    if op == "shared":
        case["batch"] = log(1, 96)
        case["groups"] = rng.choice([1, 1, rng.randint(1, min(6, case["batch"]))])
        case |= {"prefix": log(1, 32768), "prefixes": rng.choice(["full", "mixed"]), "seq": log(1, 1200), "lens": rng.choice(["full", "stairs", "mixed"])}
        case["prefix"] = min(case["prefix"], 32768 * 2048 // (heads * case["batch"] * case["groups"]))
        return case
    case |= {"sink": rng.choice([0, 1, 4, 4, 17, 128]), "window": log(1, 6000), "lens": rng.choice(["full", "stairs", "mixed"]), "cap": rng.choice(["ring", "linear"])}
    if op == "decode":
        case |= {"batch": log(1, 32), "seq": log(1, 12000) if case["cap"] == "linear" else log(1, 100000)}
        if rng.random() < 0.2:
            case |= {"dtype": "f32", "window": min(case["window"], 700), "batch": min(case["batch"], 8)}
        return case
    case |= {"batch": log(1, 16), "news": rng.choice(["full", "mixed"]), "past": log(1, 9000) - 1, "pad": rng.choice([0, 0, log(1, 100)])}
    case["new"] = log(1, max(1, 4000 // case["batch"]))
    keys = min(case["past"], case["sink"] + case["window"]) + case["new"]
    case["new"] = max(1, min(case["new"], 2 * 10 ** 9 // (heads * case["batch"] * keys)))
    return case


# ---- sizes of a case ----------------------------------------------------------------------------------------------------------


def _spread(kind, most, count, key, least=0):
    """`count` lengths up to `most`: all of them that long, one shorter than the other, or spread over the logarithm with an
    empty and a one-token sequence among them."""
    if kind == "full":
        return [most] * count
    if kind == "stairs":
        return [max(least, most - (most // 29 + 1) * b) for b in range(count)]
    r = np.random.RandomState(key)
    lens = [int(v) for v in np.exp(r.uniform(0, math.log(most + 1), count))]
    lens[0] = most
    if count > 2:
        lens[1], lens[2] = 0, 1
    return [max(least, min(most, v)) for v in lens]


def _sizes(case):
    """Lengths after the step, new tokens, rows a cache has room for."""
    op, batch = case["op"], case["batch"]
    if op == "decode":
        lens = _spread(case["lens"], case["seq"], batch, case["seq"])
        news = [min(1, n) for n in lens]
    else:
        news = _spread(case["news"], case["new"], batch, case["new"] + 1)
        past = _spread(case.get("lens", "mixed"), case.get("past", case.get("seq")), batch, case["new"] + 7)
        lens = [p + n for p, n in zip(past, news)]
    if op == "slots":
        return lens, news, case["cap_rows"]
    cap = max(lens) + 1
    if case["cap"] == "ring":
        cap = min(cap, case["sink"] + case["window"] + max(max(news), 1) + 20)
    return lens, news, (max(cap, case["sink"] + 1) + 7) // 8 * 8


def _visible(n, new, sink, window):
    """How many (query, position) pairs the last `new` tokens of a sequence of n see."""
    i = np.arange(n - new, n, dtype=np.int64)
    return int(np.where(i + 1 <= sink + window, i + 1, sink + window).sum())


def _generator(seed, tag):
    return torch.Generator(device="cuda").manual_seed(1000003 * tag + seed)


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _rows(case, width, s_cap, lens, g):
    """A cache [len(lens)][H_kv][s_cap][width] of bell-shaped rows with a few strong dimensions, as keys and values have; rows
    that nothing has been written to hold NaN."""
    gain = 1 + 2 * (torch.rand((case["kv_heads"], 1, width), generator=g, device="cuda") < 0.04).float()
    out = torch.full((len(lens), case["kv_heads"], s_cap, width), math.nan, dtype=_type(case), device="cuda")
    for b, n in enumerate(lens):
        n = min(n, s_cap)
        if n:
            out[b, :, :n] = (torch.randn((case["kv_heads"], n, width), generator=g, device="cuda") * gain).to(out.dtype)
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    return [0] + [int(v) for v in np.cumsum(counts)]


_contexts = {}


def _context(case):
    """The library context that a program keeps for a model: created once, tables built."""
    kv, heads, pairs, vch = case.get("kv_heads", 8), case.get("kv_heads", 8) * case.get("group", 4), case.get("pairs", 45), case.get("vch", 90)
    key = (heads, kv, pairs, vch, case.get("dtype"), case["batch"])
    if key not in _contexts:
        from paper_2602_02599_b200 import binding

        while len(_contexts) >= 4:
            _contexts.pop(next(iter(_contexts))).close()
        kind = binding.RAP_F32 if case.get("dtype") == "f32" else binding.RAP_BF16
        ctx = binding.RapContext(1, 1024, heads, kv, HEAD_DIM, 500000.0, binding.RAP_PAIR_HALF, kind, case["batch"], 1)
        r = np.random.RandomState(1)
        tables = [torch.empty((1, kv, n), dtype=t, device="cuda") for n, t in
                  ((HEAD_DIM // 2, torch.int32), (HEAD_DIM, torch.int32), (HEAD_DIM, torch.int32), (HEAD_DIM // 2, torch.float64))]
        ctx.rap_build_tables(r.rand(1, kv, HEAD_DIM // 2), r.rand(1, kv, HEAD_DIM), [pairs], [vch], *tables)
        torch.cuda.synchronize()
        _contexts[key] = ctx
    return _contexts[key]


def prepare(case, seed):
    op, batch, st = case["op"], case["batch"], {"case": dict(case)}
    if own:
        st["ctx"] = _context(case)
    if op == "slots":
        lens, news, _ = _sizes(case)
        order = torch.randperm(batch, generator=_generator(seed, 1), device="cuda").tolist()      # the requests in another order
        lens, news = [lens[i] for i in order], [news[i] for i in order]
        st["rows"] = sum(news) + case["pad"]
        st["past"], st["new"] = _ints([n - m for n, m in zip(lens, news)]), _ints(news)
        st["after"], st["start"] = torch.empty_like(st["past"]), torch.empty(batch + 1, dtype=torch.int32, device="cuda")
        st["seq"], st["pos"], st["slot"] = [torch.full((st["rows"],), -1, dtype=torch.int32, device="cuda") for _ in range(3)]
        return st
    w, dv, heads = 2 * case["pairs"], case["vch"], case["kv_heads"] * case["group"]
    if op == "shared":
        prefixes = _spread(case["prefixes"], case["prefix"], case["groups"], case["prefix"], least=1)
        lens = _spread(case["lens"], case["seq"], batch, case["seq"])
        cut = np.sort(np.random.RandomState(batch).randint(0, batch + 1, case["groups"] - 1))
        st["group"], st["prefix_len"] = _ints([0, *[int(c) for c in cut], batch]), _ints(prefixes)
        st["longest_prefix"] = max(prefixes)
        p_cap, s_cap = (max(prefixes) + 8) // 8 * 8, (max(lens) + 9) // 8 * 8
        st["kp"], st["vp"] = _rows(case, w, p_cap, prefixes, _generator(seed, 2)), _rows(case, dv, p_cap, prefixes, _generator(seed, 3))
        rows = batch
    else:
        lens, news, s_cap = _sizes(case)
        rows = batch if op == "decode" else sum(news) + case["pad"]
        st["start"], st["longest_new"] = _ints(_starts(news)), max(news)
    st["k"], st["v"] = _rows(case, w, s_cap, lens, _generator(seed, 4)), _rows(case, dv, s_cap, lens, _generator(seed, 5))
    st["q"] = (torch.randn((rows, heads, w), generator=_generator(seed, 6), device="cuda") * 1.4).to(_type(case))
    st["len"], st["longest"] = _ints(lens), max(lens)
    # where the outputs go: rows behind the last sequence's stay as they are
    st["out"] = torch.ones((rows, heads, dv), dtype=torch.float32, device="cuda")
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------------------


def _row_of(pos, sink, s_cap):
    """The cache row of a position."""
    return torch.where(pos < sink, pos, sink + (pos - sink) % (s_cap - sink))


def _gather(cache, rows):
    """cache [B][H_kv][S_cap][W], rows [B][M] -> fp32 [B][H_kv][M][W]."""
    at = rows.long()[:, None, :, None].expand(-1, cache.shape[1], -1, cache.shape[3])
    return cache.gather(2, at).float()


def _attend(q, k, v, seen):
    """q [..., N, W], k [..., M, W], v [..., M, dv], seen [..., N, M]: (sums of weight times v, sums of weights, largest
    logits), the weights relative to the largest."""
    logits = (q @ k.transpose(-1, -2) * (1 / math.sqrt(HEAD_DIM))).masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(logits.sub_(top))
    return p @ v, p.sum(-1, keepdim=True), top


def _divided(o, total):
    return torch.where(total > 0, o / total, 0.0)


def _decode(st):
    case, lens = st["case"], st["len"]
    sink, window, s_cap = case["sink"], case["window"], st["k"].shape[2]
    if own:
        st["ctx"].rap_decode_attn_window(0, case["batch"], st["q"], st["k"], st["v"], s_cap, lens, st["longest"], sink, window, st["out"])
        return st["out"]
    m = torch.arange(min(sink + window, max(1, st["longest"])), device=lens.device)
    first = (lens - window).clamp_min(sink)[:, None]
    pos = torch.where(m < sink, m, first + m - sink)                  # [B][M]
    seen = pos < lens[:, None]
    rows = _row_of(torch.where(seen, pos, 0), sink, s_cap)
    k, v = _gather(st["k"], rows), _gather(st["v"], rows).masked_fill(~seen[:, None, :, None], 0.0)
    q = st["q"].float().unflatten(1, (case["kv_heads"], case["group"]))
    o, total, _ = _attend(q, k, v, seen[:, None, None, :])
    return _divided(o, total).flatten(1, 2)


def _prefill(st):
    case, lens, start = st["case"], st["len"], st["start"]
    sink, window, s_cap = case["sink"], case["window"], st["k"].shape[2]
    batch, kv, group, n_rows = case["batch"], case["kv_heads"], case["group"], st["q"].shape[0]
    if own:
        st["ctx"].rap_prefill_attn_window(0, batch, n_rows, st["q"], st["k"], st["v"], s_cap, start, lens, st["longest_new"], st["longest"],
                                          sink, window, st["out"])
        return st["out"]
    most = max(1, st["longest_new"])
    begin = lens - (start[1:] - start[:-1])
    m = torch.arange(min(sink + window - 1 + most, max(1, st["longest"])), device=lens.device)
    first = (begin - window + 1).clamp_min(sink)[:, None]
    pos = torch.where(m < sink, m, first + m - sink)                  # [B][M]
    there = pos < lens[:, None]
    rows = _row_of(torch.where(there, pos, 0), sink, s_cap)
    k, v = _gather(st["k"], rows), _gather(st["v"], rows).masked_fill(~there[:, None, :, None], 0.0)
    i = torch.arange(most, device=lens.device)
    at = (begin[:, None] + i)[:, :, None]                             # positions of the queries
    seen = there[:, None, :] & (pos[:, None, :] <= at) & ((pos[:, None, :] < sink) | (pos[:, None, :] > at - window))
    q = st["q"][(start[:-1, None] + i).clamp_max(n_rows - 1).long()].float()
    q = q.unflatten(2, (kv, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)              # [B][H_kv][new * G][W]
    o, total, _ = _attend(q, k, v, seen.repeat_interleave(group, 1)[:, None])
    o = _divided(o, total).unflatten(2, (most, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    r = torch.arange(n_rows, device=lens.device, dtype=torch.int32)
    b = torch.bucketize(r, start[1:], right=True).clamp_max(batch - 1)
    mine = (r - start[b]).clamp_max(most - 1).long()
    return torch.where((r < start[-1])[:, None, None], o[b, mine], st["out"])


def _shared(st):
    case, lens, first = st["case"], st["len"], st["group"]
    batch, kv, group = case["batch"], case["kv_heads"], case["group"]
    if own:
        st["ctx"].rap_decode_attn_shared(0, batch, st["q"], case["groups"], st["kp"], st["vp"], st["kp"].shape[2], first, st["prefix_len"],
                                         st["longest_prefix"], st["k"], st["v"], st["k"].shape[2], lens, st["longest"], st["out"])
        return st["out"]
    q = st["q"].float().unflatten(1, (kv, group))
    # the prefixes, each with all its sequences' queries at once
    place = torch.arange(batch, device=lens.device)
    n = torch.bucketize(place, first[1:], right=True)
    at = (first[:-1, None] + torch.arange(batch, device=lens.device)).clamp_max(batch - 1).long()     # [N][B]
    qg = q[at].permute(0, 2, 1, 3, 4).flatten(2, 3)                                                  # [N][H_kv][B * G][W]
    there = (torch.arange(st["kp"].shape[2], device=lens.device) < st["prefix_len"][:, None])[:, None, None, :]
    vp = st["vp"].float().masked_fill_(~there.transpose(-1, -2), 0.0)
    parts = _attend(qg, st["kp"].float(), vp, there)
    at = place - first[n]
    o1, s1, m1 = [x.unflatten(2, (batch, group))[n, :, at.long()] for x in parts]
    # every sequence's own rows
    there = (torch.arange(st["k"].shape[2], device=lens.device) < lens[:, None])[:, None, None, :]
    v = st["v"].float().masked_fill_(~there.transpose(-1, -2), 0.0)
    o2, s2, m2 = _attend(q, st["k"].float(), v, there)
    top = torch.maximum(m1, m2)
    f1, f2 = torch.exp(m1 - top), torch.exp(m2 - top)
    return _divided(o1 * f1 + o2 * f2, s1 * f1 + s2 * f2).flatten(1, 2)


def _slots(st):
    case, past, new = st["case"], st["past"], st["new"]
    if own:
        st["ctx"].rap_build_slots(case["batch"], past, new, None, st["rows"], case["sink"], case["cap_rows"], st["start"], st["seq"], st["pos"],
                                  st["slot"], st["after"])
        return st["start"], st["seq"], st["pos"], st["slot"], st["after"]
    start = torch.nn.functional.pad(torch.cumsum(new, 0), (1, 0)).int()
    r = torch.arange(st["rows"], device=past.device, dtype=torch.int32)
    b = torch.bucketize(r, start[1:], right=True).clamp_max(case["batch"] - 1)
    pos = past[b] + r - start[b]
    mine = r < start[-1]
    slot = _row_of(pos, case["sink"], case["cap_rows"])
    return start, torch.where(mine, b.int(), st["seq"]), torch.where(mine, pos, st["pos"]), torch.where(mine, slot, st["slot"]), past + new


def run(state):
    return {"decode": _decode, "prefill": _prefill, "shared": _shared, "slots": _slots}[state["case"]["op"]](state)


def work(case):
    op, batch = case["op"], case["batch"]
    if op == "slots":
        _, news, _ = _sizes(case)
        return {"bytes": 4 * (4 * batch + 1 + 3 * sum(news)), "flops": 0}
    w, heads, e = 2 * case["pairs"] + case["vch"], case["kv_heads"] * case["group"], 4 if case["dtype"] == "f32" else 2
    if op == "shared":
        prefixes = _spread(case["prefixes"], case["prefix"], case["groups"], case["prefix"], least=1)
        lens = _spread(case["lens"], case["seq"], batch, case["seq"])
        cut = np.sort(np.random.RandomState(batch).randint(0, batch + 1, case["groups"] - 1))
        edge = [0, *[int(c) for c in cut], batch]
        read = sum(p for n, p in enumerate(prefixes) if edge[n + 1] > edge[n]) + sum(lens)
        pairs = sum(p * (edge[n + 1] - edge[n]) for n, p in enumerate(prefixes)) + sum(lens)
        rows = batch
    else:
        lens, news, _ = _sizes(case)
        sink, window = case["sink"], case["window"]
        read = sum(min(n, sink + window + m - 1) for n, m in zip(lens, news) if m)
        pairs = sum(_visible(n, m, sink, window) for n, m in zip(lens, news))
        rows = batch if op == "decode" else sum(news)
    return {"bytes": read * case["kv_heads"] * w * e + rows * heads * (2 * case["pairs"] * e + 4 * case["vch"]), "flops": max(1, 2 * pairs * heads * w)}


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------


def exact(case, seed):
    global own
    was, own = own, False      # the inputs alone
    try:
        st = prepare(case, seed)
    finally:
        own = was
    op, batch = case["op"], case["batch"]
    if op == "slots":
        past, new = st["past"].tolist(), st["new"].tolist()
        start, after = np.zeros(batch + 1, np.int32), np.array(past, np.int32) + np.array(new, np.int32)
        seq, pos, slot = [np.full(st["rows"], -1, np.int32) for _ in range(3)]
        r, sink = 0, case["sink"]
        for b in range(batch):
            for p in range(past[b], past[b] + new[b]):
                seq[r], pos[r], slot[r] = b, p, p if p < sink else sink + (p - sink) % (case["cap_rows"] - sink)
                r += 1
            start[b + 1] = r
        return start, seq, pos, slot, after
    kv, group = case["kv_heads"], case["group"]
    out = st["out"].double()
    q = st["q"].double()
    lens = st["len"].tolist()
    if op == "shared":
        edge, prefixes = st["group"].tolist(), st["prefix_len"].tolist()
        for n in range(case["groups"]):
            for b in range(edge[n], edge[n + 1]):
                for h in range(kv):
                    k = torch.cat([st["kp"][n, h, :prefixes[n]], st["k"][b, h, :lens[b]]]).double()
                    v = torch.cat([st["vp"][n, h, :prefixes[n]], st["v"][b, h, :lens[b]]]).double()
                    out[b, h * group: (h + 1) * group] = torch.softmax(q[b, h * group: (h + 1) * group] @ k.T / math.sqrt(HEAD_DIM), -1) @ v
        return out
    sink, window, s_cap = case["sink"], case["window"], st["k"].shape[2]
    _, news, _ = _sizes(case)
    first = 0
    for b, n in enumerate(lens):
        if op == "decode":
            first, m = b, 1
        else:
            m = news[b]
        if n == 0 and m:
            out[first] = 0
        elif m:
            old = max(0, n - m - window + 1)      # the oldest position that one of them sees behind the sinks
            pos = torch.tensor(list(range(min(sink, old))) + list(range(old, n)), device="cuda")
            row = torch.tensor([p if p < sink else sink + (p - sink) % (s_cap - sink) for p in pos.tolist()], device="cuda")
            for h in range(kv):
                k, v = st["k"][b, h][row].double(), st["v"][b, h][row].double()
                for c in range(0, m, 2048):       # in pieces: 64-bit logits of a long block are large
                    i = torch.arange(n - m, n, device="cuda")[c: c + 2048, None]
                    hidden = (pos > i) | ((pos >= sink) & (pos <= i - window))
                    here = slice(first + c, first + c + len(i))
                    logits = torch.einsum("tgw,jw->gtj", q[here, h * group: (h + 1) * group], k) / math.sqrt(HEAD_DIM)
                    p = torch.softmax(logits.masked_fill(hidden, -math.inf), -1)
                    out[here, h * group: (h + 1) * group] = torch.einsum("gtj,jd->tgd", p, v)
        first += m
    return out
