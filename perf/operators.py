"""What a server of dense and sparse decode calls around a paged cache, as cases that can be timed: the rows of a step and
where they go, rotary positions with the cache write, attention of new rows over the cache, and attention of a batch that
shares a prefix.

A case is a dict of plain values.  `prepare` makes on the GPU what a program holds before the call.  `run` is one pass: in
plain torch operations in 32 bits (angles of rotary positions in 64) where `own` is false, through the binding's entry
points where it is true; `exact` gives the same values in 64 bits from the definition.  Kinds:

  map     absb_map_rows: from the requests' lengths before and after a step, the rows of the step, their positions and
          slots, and the page table with pages taken from a ring of free ones or given back to it
  rotate  absb_rotate_store: rotary positions for queries and keys, and keys and values into the paged cache
  attend  absb_attend_rows: attention of every request's new rows over its context, with a tanh cap, a distance bias, a
          window, document starts, prefixes seen by all rows
  shared  absb_attend_shared: the same where groups of requests share their first pages

Ranges that the cases stand for (`draw` spreads over them): contexts of one token to 128 Ki, 1 to 64 requests (map: 1024)
of equal or ragged lengths, 1 to 8192 new rows a request (rotate: 32 Ki in all), 1 to 16 KV heads in groups of 1 to 8, f16 and
bf16, pages of 8 to 128 tokens, pages head by head or token by token, prefixes of no pages to 64 Ki tokens.
"""
import math
import random

import numpy as np
import torch

own = False

D = 128  # head dimension
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}


def case(**kw):
    """A case with the defaults of a Llama-3.1-8B-shaped layer.  Lengths are drawn from [len_lo, len_hi] and new rows from
    [new_lo, new_hi], per request, by `shape_seed` (shapes belong to the case, values to the seed)."""
    c = dict(kind="attend", dtype="f16", batch=1, q_heads=32, kv_heads=8, page=64, order="hnd", len_lo=4096, len_hi=4096,
             new_lo=1, new_hi=1, shape_seed=1, softcap=0.0, bias=False, window=0, docs=0, prefix_pct=0, groups=1, shared=0,
             finish_pct=0, join_pct=0, pairs=False, rot=128, base=500000.0, factor=1.0)
    c.update(kw)
    return c


def listed():
    return [
        # a decode step's bookkeeping: every request grows by one token; launch latency is all there is
        case(name="map_decode_b64", kind="map", batch=64, len_lo=100, len_hi=32768),
        # a busy scheduler step: requests that finish, prompts that join, small pages
        case(name="map_mixed_b512", kind="map", batch=512, page=16, len_lo=1, len_hi=16384, new_lo=1, new_hi=2048, finish_pct=20,
             join_pct=30),
        # the new tokens of a ragged serving batch at far positions, five query heads per KV head
        case(name="rotate_decode_b16", kind="rotate", dtype="bf16", batch=16, q_heads=40, len_lo=8192, len_hi=131072),
        # the prompt of one 8K request
        case(name="rotate_prompt_8k", kind="rotate", len_lo=8192, len_hi=8192, new_lo=8192, new_hi=8192),
        # a packed batch of long chunks, neighbours rotated, half of the head, positions stretched eightfold, token-major pages
        case(name="rotate_chunks_pairs", kind="rotate", dtype="bf16", batch=4, order="nhd", page=16, len_lo=60001, len_hi=120001,
             new_lo=8001, new_hi=8191, pairs=True, rot=64, base=10000.0, factor=8.0),
        # the prompt of one request, nothing but the causal order
        case(name="attend_prompt_4k", new_lo=4096, new_hi=4096),
        # chunks of ragged prompts behind long contexts, capped scores in a window
        case(name="attend_chunk_cap_b4", dtype="bf16", batch=4, len_lo=8000, len_hi=16000, new_lo=301, new_hi=1023, softcap=50.0,
             window=4096),
        # single tokens of a ragged batch, distance bias
        case(name="attend_token_bias_b8", batch=8, len_lo=4000, len_hi=32768, bias=True),
        # one packed row of documents, five query heads per KV head
        case(name="attend_docs_8k", dtype="bf16", q_heads=40, page=32, len_lo=8192, len_hi=8192, new_lo=8192, new_hi=8192, docs=12),
        # a short system prompt before a few short chats
        case(name="shared_4k_b8", kind="shared", dtype="bf16", batch=8, shared=4096, len_lo=17, len_hi=300),
        # a long document asked about by many
        case(name="shared_32k_b64", kind="shared", batch=64, shared=32768, len_lo=1, len_hi=1000),
        # two prefixes, capped scores, a few new rows each
        case(name="shared_two_cap_b40", kind="shared", dtype="bf16", batch=40, groups=2, shared=8192, len_lo=9, len_hi=2000,
             new_lo=1, new_hi=8, softcap=30.0, page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_SCORES, MOST_GATHERED, MOST_ROTATED = 2.7e9, 17.5e6, 32768 * 48


def draw(rng):
    while True:
        kind = rng.choices(("map", "rotate", "attend", "shared"), (1, 2, 5, 3))[0]
        kv = rng.choices((1, 2, 4, 8, 16), (1, 1, 2, 6, 1))[0]
        c = case(kind=kind, dtype=rng.choice(("f16", "bf16")), kv_heads=kv, q_heads=kv * rng.choice((1, 2, 3, 4, 4, 5, 6, 7, 8)),
                 page=rng.choice((8, 16, 32, 64, 64, 128)), order=rng.choice(("hnd", "hnd", "nhd")), shape_seed=rng.randrange(1 << 20),
                 batch=_log(rng, 1, 1024 if kind == "map" else 64))
        hi = _log(rng, 1, 131072)
        c["len_hi"], c["len_lo"] = hi, hi if rng.random() < 0.4 else max(1, int(hi * rng.uniform(0.05, 0.9)))
        new = 1 if rng.random() < 0.4 else _log(rng, 1, 8192)
        c["new_hi"], c["new_lo"] = new, new if rng.random() < 0.4 else max(1, int(new * rng.uniform(0.05, 0.9)))
        if kind == "map":
            c["finish_pct"], c["join_pct"] = rng.choice((0, 10, 30)), rng.choice((0, 10, 30))
        elif kind == "rotate":
            c["pairs"], c["rot"] = rng.random() < 0.4, rng.choice((128, 128, 128, 64, 96, 32, 2))
            c["base"], c["factor"] = rng.choice((10000.0, 500000.0, 1000000.0)), rng.choice((1.0, 1.0, 4.0, 8.0))
        else:
            c["softcap"] = rng.choice((0.0, 0.0, 30.0, 50.0))
            c["bias"] = rng.random() < 0.25
            c["window"] = rng.choice((0, 0, 0, _log(rng, 1, 8192)))
            if kind == "attend":
                c["docs"] = rng.choice((0, 0, _log(rng, 1, 40)))
                c["prefix_pct"] = rng.choice((0, 0, 0, 30, 100))
            else:
                c["groups"] = rng.choice((1, 1, 2, 3))
                c["shared"] = c["page"] * rng.choice((0, _log(rng, 1, 65536 // c["page"])))
                c["new_hi"], c["new_lo"] = min(c["new_hi"], 64), min(c["new_lo"], 64)
        n, lens, _ = shapes(c)
        if kind == "map":
            if lens.sum() > 4e6:
                continue
        elif kind == "rotate":
            if n.sum() * (c["q_heads"] + 2 * kv) > MOST_ROTATED:
                continue
        elif c["batch"] * c["q_heads"] * int(n.max()) * int(lens.max()) > MOST_SCORES or c["batch"] * int(lens.max()) * kv > MOST_GATHERED:
            continue
        if kind != "map" and not n.sum():
            continue
        return c


# ------------------------------------------------------------------ shapes of a case
def shapes(c):
    """(new rows, lengths after the step, shared tokens) of every request."""
    r = random.Random(c["shape_seed"])
    B = c["batch"]
    lens = np.array([r.randint(c["len_lo"], c["len_hi"]) for _ in range(B)], np.int64)
    new = np.array([r.randint(c["new_lo"], c["new_hi"]) for _ in range(B)], np.int64)
    if c["kind"] == "map":
        what = [r.randrange(100) for _ in range(B)]
        return new, lens, np.array([-1 if w < c["finish_pct"] else 1 if w < c["finish_pct"] + c["join_pct"] else 0 for w in what])
    if c["kind"] == "shared":
        first = group_starts(c)
        group = np.repeat(np.arange(c["groups"]), np.diff(first))
        # the first group's prefix has the case's length, the others half of the one before
        pre = (np.array([c["shared"] >> g for g in range(c["groups"])], np.int64) // c["page"]) * c["page"]
        lens = np.maximum(lens, new) + pre[group]
        return new, lens, pre
    return np.minimum(new, lens), lens, np.zeros(1, np.int64)


def group_starts(c):
    return np.array([c["batch"] * g // c["groups"] for g in range(c["groups"] + 1)], np.int64)


def before_after(c):
    """Lengths of a map case's requests before and after the step."""
    new, lens, what = shapes(c)
    before = np.where(what == 1, 0, lens)
    after = np.where(what == -1, 0, np.where(what == 1, new, lens + 1))
    return before, after


def documents(c):
    """First token of the document that every row of an attend case belongs to."""
    r = random.Random(c["shape_seed"] + 5)
    new, lens, _ = shapes(c)
    got = []
    for n, L in zip(new.tolist(), lens.tolist()):
        starts = np.array(sorted({0} | {r.randrange(L) for _ in range(c["docs"])}))
        rows = np.arange(L - n, L)
        got.append(starts[np.searchsorted(starts, rows, side="right") - 1])
    return np.concatenate(got).astype(np.int32)


def prefixes(c):
    new, lens, _ = shapes(c)
    return (lens * c["prefix_pct"] // 100).astype(np.int32)


def intervals(c):
    """First and last key that every row sees, request after request, and the row's own position."""
    new, lens, _ = shapes(c)
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new.tolist(), lens.tolist())])
    lo = np.zeros_like(pos)
    if c["window"]:
        lo = np.maximum(lo, pos - c["window"] + 1)
    if c["docs"]:
        lo = np.maximum(lo, documents(c))
    hi = pos
    if c["prefix_pct"]:
        hi = np.maximum(pos, np.repeat(prefixes(c).astype(np.int64), new) - 1)
    return lo, hi, pos


def work(c):
    """Of one pass.  map: lengths in, rows and table entries out.  rotate: queries, keys, values, positions and slots in,
    queries and cache rows out.  attend, shared: queries in, outputs and log-sums out, every key and value that some row
    of the request sees once (a shared one once for the group), 4 d operations for every visible (query head, key)."""
    if c["kind"] == "map":
        before, after = before_after(c)
        P = c["page"]
        moved = np.abs(-(-after // P) + before // -P).sum()
        rows = np.maximum(after - before, 0).sum()
        return {"bytes": float(8 * c["batch"] + 4 * (c["batch"] + 1) + 12 * rows + 8 * moved), "flops": float(rows + moved)}
    new, lens, pre = shapes(c)
    rows, Hq, Hkv = float(new.sum()), c["q_heads"], c["kv_heads"]
    if c["kind"] == "rotate":
        return {"bytes": rows * ((2 * Hq + 4 * Hkv) * 2 * D + 12), "flops": rows * (Hq + Hkv) * 3.0 * c["rot"]}
    lo, hi, _ = intervals(c)
    seen = np.maximum(hi - lo + 1, 0)
    keys = 0.0
    start = np.concatenate([[0], np.cumsum(new)])
    if c["kind"] == "attend":
        for b in range(c["batch"]):
            rlo, rhi = lo[start[b]:start[b + 1]], hi[start[b]:start[b + 1]]
            keys += max(0, rhi.max() - rlo.min() + 1) if len(rlo) else 0
    else:
        first = group_starts(c)
        for g in range(c["groups"]):
            low = [lo[start[b]:start[b + 1]].min() for b in range(first[g], first[g + 1])]
            keys += max(0, int(pre[g]) - min(low)) if low else 0
            keys += sum(int(lens[b]) - max(int(pre[g]), low[b - first[g]]) for b in range(first[g], first[g + 1]))
    return {"bytes": float(rows * Hq * (4 * D + 4) + keys * Hkv * 4 * D), "flops": float(seen.sum()) * Hq * 4 * D}


# ------------------------------------------------------------------ what a program has in hand before the call
def _tables(c, g, lens, pre):
    """A page table over shuffled pages, requests of a group on the same first pages; and how many pages there are."""
    P, B = c["page"], c["batch"]
    n = -(-lens // P)
    table = np.zeros((B, int(n.max())), np.int64)
    at = 0
    if c["kind"] == "shared":
        first = group_starts(c)
        for j in range(c["groups"]):
            m = int(pre[j]) // P
            for b in range(first[j], first[j + 1]):
                table[b, :m] = np.arange(at, at + m)
            at += m
            for b in range(first[j], first[j + 1]):
                table[b, m:n[b]] = np.arange(at, at + n[b] - m)
                at += int(n[b]) - m
    else:
        for b in range(B):
            table[b, :n[b]] = np.arange(at, at + n[b])
            at += int(n[b])
    perm = torch.randperm(max(at, 1), generator=g, device="cuda").int()
    return perm[torch.from_numpy(table).cuda()], max(at, 1)


def _cache(c, g, pages):
    """[page][head][slot][channel], in memory head by head or token by token."""
    x = torch.randn((pages, c["kv_heads"], c["page"], D) if c["order"] == "hnd" else (pages, c["page"], c["kv_heads"], D),
                    generator=g, device="cuda").to(TORCH[c["dtype"]])
    return x if c["order"] == "hnd" else x.transpose(1, 2)


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()  # noqa: E731
    s = {"case": c}
    if c["kind"] == "map":
        before, after = before_after(c)
        P = c["page"]
        had, need = -(-before // P), -(-after // P)
        width = int(max(had.max(), need.max(), 1))
        taken, free = int(had.sum()), int(np.maximum(need - had, 0).sum()) + 100
        perm = torch.randperm(taken + free, generator=g, device="cuda").int()
        table = np.full((c["batch"], width), taken + free, np.int64)
        mine = np.arange(width)[None, :] < had[:, None]
        table[mine] = np.arange(taken)
        perm1 = torch.cat([perm, torch.full((1,), -1, dtype=torch.int32, device="cuda")])
        s["page_table"] = perm1[torch.from_numpy(table).cuda()]
        # the ring of free pages: as many places as there are pages, the free ones from some place on
        head = int(torch.randint(0, taken + free, (1,), generator=g, device="cuda"))
        ring = torch.zeros(taken + free, dtype=torch.int32, device="cuda")
        ring[(head + torch.arange(free, device="cuda")) % (taken + free)] = perm[taken:]
        s["ring"] = ring
        s["cursors"] = torch.tensor([head, head + free, 0, 0], dtype=torch.int64, device="cuda")
        s["before"], s["after"], s["after_host"] = i32(before), i32(after), after.astype(np.int32)
        s["rows"] = int(np.maximum(after - before, 0).sum())
        return s
    new, lens, pre = shapes(c)
    tdt = TORCH[c["dtype"]]
    Hq, Hkv = c["q_heads"], c["kv_heads"]
    off = np.concatenate([[0], np.cumsum(new)])
    rows = int(off[-1])
    if c["kind"] == "rotate":
        # pages of the new tokens alone: what else a context holds does not matter to the call
        P, pos = c["page"], intervals(c)[2]
        first = (lens - new) // P
        count = (lens - 1) // P + 1 - first
        base = np.repeat(np.cumsum(count) - count - first, new)
        pages = int(count.sum())
        perm = torch.randperm(pages, generator=g, device="cuda")
        s["row_pos"] = i32(pos)
        s["row_slot"] = perm[torch.from_numpy(base + pos // P).cuda()] * P + torch.from_numpy(pos % P).cuda()
        s["k_cache"], s["v_cache"] = _cache(c, g, pages), _cache(c, g, pages)
        # queries, keys and values side by side, as one projection gives them
        s["qkv"] = torch.randn((rows, (Hq + 2 * Hkv) * D), generator=g, device="cuda").to(tdt)
        freq = c["base"] ** (-np.arange(0, c["rot"], 2, dtype=np.float64) / c["rot"]) / c["factor"]
        s["freq"] = torch.from_numpy(freq).cuda()
        s["q_out"] = torch.empty((rows, Hq, D), dtype=tdt, device="cuda")
        return s
    s["page_table"], pages = _tables(c, g, lens, pre)
    s["k_cache"], s["v_cache"] = _cache(c, g, pages), _cache(c, g, pages)
    s["lens"], s["lens_host"] = i32(lens), lens.astype(np.int32)
    s["row_off"], s["row_off_host"] = i32(off), off.astype(np.int32)
    s["q"] = (1.5 * torch.randn((rows, Hq, D), generator=g, device="cuda")).to(tdt)
    s["slopes"] = s["doc_start"] = s["prefix"] = None
    if c["bias"]:
        s["slopes"] = torch.from_numpy(np.exp2(-8.0 * np.arange(1, Hq + 1) / Hq).astype(np.float32)).cuda()
    if c["docs"]:
        s["doc_start"] = i32(documents(c))
    if c["prefix_pct"]:
        s["prefix"] = i32(prefixes(c))
    if c["kind"] == "shared":
        s["first_host"], s["shared_host"] = group_starts(c).astype(np.int32), pre.astype(np.int32)
        s["first"], s["shared"] = i32(s["first_host"]), i32(pre)
    s["out"] = torch.empty((rows, Hq, D), dtype=tdt, device="cuda")
    s["lse"] = torch.empty((rows, Hq), dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass, plain
def _map_plain(s):
    c, before, after, table, ring = s["case"], s["before"].long(), s["after"].long(), s["page_table"], s["ring"]
    P, cap = c["page"], len(s["ring"])
    head, tail = s["cursors"][0], s["cursors"][1]
    off = torch.nn.functional.pad(torch.cumsum(torch.clamp(after - before, min=0), 0), (1, 0))
    had, need = (before + P - 1) // P, (after + P - 1) // P
    take, give = torch.clamp(need - had, min=0), torch.clamp(had - need, min=0)
    take_at, give_at = torch.cumsum(take, 0) - take, torch.cumsum(give, 0) - give
    missing = torch.clamp(take.sum() - (tail - head), min=0)
    fine = missing == 0
    col = torch.arange(table.shape[1], device=table.device)[None]
    fresh = ring[(head + take_at[:, None] + col - had[:, None]) % cap]
    new_table = torch.where((col >= had[:, None]) & (col < need[:, None]) & fine, fresh, table)
    given = (col >= need[:, None]) & (col < had[:, None]) & fine
    place = torch.where(given, (tail + give_at[:, None] + col - need[:, None]) % cap, cap)
    new_ring = torch.nn.functional.pad(ring, (0, 1)).scatter(0, place.reshape(-1), table.reshape(-1))[:cap]
    rows = torch.arange(s["rows"], device=table.device)
    req = torch.searchsorted(off[1:], rows, right=True)
    pos = before[req] + rows - off[req]
    slot = torch.where(fine, new_table[req, pos // P].long() * P + pos % P, -1)
    moved = torch.stack([take.sum(), give.sum()]) * fine
    cursors = torch.cat([s["cursors"][:2] + moved, missing[None], torch.zeros_like(head)[None]])
    return {"row_off": off.int(), "row_pos": pos.int(), "row_slot": slot, "page_table": new_table, "ring": new_ring, "cursors": cursors}


def _turn(x, cos, sin, pairs, rot):
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if pairs else (r[..., :rot // 2], r[..., rot // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    r = torch.stack([a, b], -1).flatten(-2) if pairs else torch.cat([a, b], -1)
    return torch.cat([r, rest], -1)


def _rotate_plain(s):
    c = s["case"]
    Hq, Hkv, P = c["q_heads"], c["kv_heads"], c["page"]
    q, k, v = s["qkv"].view(-1, Hq + 2 * Hkv, D).split((Hq, Hkv, Hkv), 1)
    angle = (s["row_pos"].double()[:, None] * s["freq"])[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    page, slot = s["row_slot"] // P, s["row_slot"] % P
    s["q_out"].copy_(_turn(q, cos, sin, c["pairs"], c["rot"]))
    s["k_cache"][page, :, slot] = _turn(k, cos, sin, c["pairs"], c["rot"]).to(s["k_cache"].dtype)
    s["v_cache"][page, :, slot] = v
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend_plain(s):
    c, q, table = s["case"], s["q"], s["page_table"].long()
    Hq, Hkv, P, B = c["q_heads"], c["kv_heads"], c["page"], c["batch"]
    G, n, L = Hq // Hkv, int(np.diff(s["row_off_host"]).max()), int(s["lens_host"].max())
    lens, off = s["lens"].long(), s["row_off"].long()
    j = torch.arange(L, device=q.device)
    page = table[:, j // P]  # (beyond a context: any page, masked below)
    k = s["k_cache"][page, :, j % P].float().permute(0, 2, 3, 1)  # [B][Hkv][d][L]
    v = s["v_cache"][page, :, j % P].float().permute(0, 2, 1, 3)  # [B][Hkv][L][d]
    at = torch.arange(n, device=q.device)[None] + off[:-1, None]  # rows of every request, beyond its last: repeated
    count = (off[1:] - off[:-1])[:, None]
    at = torch.minimum(at, torch.clamp(off[1:, None] - 1, min=0))
    i = (lens[:, None] - count + torch.arange(n, device=q.device)[None])[:, :, None]
    rows = q[at].float().view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    x = (torch.matmul(rows, k) / math.sqrt(D)).view(B, Hkv, n, G, L)
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    if s["slopes"] is not None:
        x = x - s["slopes"].view(1, Hkv, 1, G, 1) * (i - j).abs().float()[:, None, :, None]
    seen = j <= i
    if s["prefix"] is not None:
        seen = seen | (j < s["prefix"][:, None, None])
    if c["window"]:
        seen = seen & (i - j < c["window"])
    if s["doc_start"] is not None:
        seen = seen & (j >= s["doc_start"][at][:, :, None])
    seen = seen & (j < lens[:, None, None])
    x = x.masked_fill(~seen[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    out = torch.matmul(e.view(B, Hkv, n * G, L), v).view(B, Hkv, n, G, D) / torch.where(total == 0, 1.0, total)
    lse = (top + torch.log(total)).squeeze(-1)
    req = torch.searchsorted(off[1:].contiguous(), torch.arange(len(q), device=q.device), right=True)
    nth = torch.arange(len(q), device=q.device) - off[req]
    s["out"].copy_(out.permute(0, 2, 1, 3, 4)[req, nth].view(-1, Hq, D))
    s["lse"].copy_(lse.permute(0, 2, 1, 3)[req, nth].view(-1, Hq))
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------ one pass, through the framework
def _program(s):
    """What a serving program keeps beside its tensors: the binding's records, a workspace, result buffers."""
    from paper_2605_12110_amd import absb
    c = s["case"]
    P, Hkv, dt = c["page"], c["kv_heads"], {"f16": absb.F16, "bf16": absb.BF16}[c["dtype"]]
    strides = (Hkv * P * D, P * D, D) if c["order"] == "hnd" else (P * Hkv * D, D, Hkv * D)
    layer = absb.Layer(c["q_heads"], Hkv, D, P, dt, None, strides)
    p = {"absb": absb, "layer": layer}
    if c["kind"] == "map":
        p["batch"] = absb.Batch(seq_lens_host=s["after_host"], seq_lens=s["after"], page_table=s["page_table"])
        p["ring"] = absb.PageRing(s["ring"], s["cursors"])
        new = lambda n, t: torch.zeros(n, dtype=t, device="cuda")  # noqa: E731
        p["out"] = (new(c["batch"] + 1, torch.int32), new(s["rows"], torch.int32), new(s["rows"], torch.int64))
        p["cursors"] = new(4, torch.int64)
        return p
    if c["kind"] == "rotate":
        p["rope"] = absb.Rope(rot_dim=c["rot"], layout=absb.ROPE_PAIRS if c["pairs"] else absb.ROPE_HALVES)
        p["qkv"] = s["qkv"].view(-1, c["q_heads"] + 2 * Hkv, D).split((c["q_heads"], Hkv, Hkv), 1)
        return p
    p["batch"] = absb.Batch(seq_lens_host=s["lens_host"], seq_lens=s["lens"], page_table=s["page_table"])
    p["rows"] = absb.Rows(s["row_off_host"], s["row_off"])
    p["opts"] = absb.ScoreOpts(softcap=c["softcap"], slopes=s["slopes"], window=c["window"], prefix_lens=s["prefix"],
                               doc_start=s["doc_start"])
    p["shared"] = None
    if c["kind"] == "shared":
        p["shared"] = absb.SharedPrefix(s["first_host"], s["shared_host"], s["first"], s["shared"])
    p["workspace"] = torch.zeros(absb.absb_attend_workspace(layer, p["batch"], p["rows"], p["shared"]), dtype=torch.uint8, device="cuda")
    return p


def _run_own(s):
    p = s.get("program")
    if p is None:
        p = s["program"] = _program(s)
    absb, kind = p["absb"], s["case"]["kind"]
    if kind == "map":
        off, pos, slot = p["out"]
        absb.absb_map_rows(p["layer"], p["batch"], s["before"], s["page_table"], off, pos, slot, p["ring"], p["cursors"])
        return {"row_off": off, "row_pos": pos, "row_slot": slot, "page_table": s["page_table"], "ring": s["ring"], "cursors": p["cursors"]}
    if kind == "rotate":
        q, k, v = p["qkv"]
        absb.absb_rotate_store(p["layer"], p["rope"], s["row_pos"], s["row_slot"], s["freq"], q, s["q_out"], k, v, s["k_cache"], s["v_cache"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if kind == "attend":
        absb.absb_attend_rows(p["layer"], p["batch"], p["rows"], s["q"], s["k_cache"], s["v_cache"], s["out"], s["lse"], p["opts"], p["workspace"])
    else:
        absb.absb_attend_shared(p["layer"], p["batch"], p["rows"], p["shared"], s["q"], s["k_cache"], s["v_cache"], s["out"], s["lse"],
                                p["opts"], p["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    return _map_plain(s) if kind == "map" else _rotate_plain(s) if kind == "rotate" else _attend_plain(s)


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(c, seed):
    if c["kind"] == "map":
        return None  # whole numbers throughout
    s = prepare(c, seed)
    Hq, Hkv, P = c["q_heads"], c["kv_heads"], c["page"]
    G = Hq // Hkv
    if c["kind"] == "rotate":
        x = s["qkv"].double().view(-1, Hq + 2 * Hkv, D)
        turned = x[:, :Hq + Hkv].clone()
        half = c["rot"] // 2
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if c["pairs"] else (i, i + half)
            t = torch.polar(torch.ones(len(x), dtype=torch.float64, device="cuda"), s["row_pos"].double() * s["freq"][i])
            z = torch.complex(x[:, :Hq + Hkv, a], x[:, :Hq + Hkv, b]) * t[:, None]
            turned[:, :, a], turned[:, :, b] = z.real, z.imag
        k, v = s["k_cache"].double(), s["v_cache"].double()
        page, slot = torch.div(s["row_slot"], P, rounding_mode="floor"), s["row_slot"] % P
        k[page, :, slot], v[page, :, slot] = turned[:, Hq:], x[:, Hq + Hkv:]
        return {"q": turned[:, :Hq], "k_cache": k, "v_cache": v}
    lo, hi, pos = (torch.from_numpy(a).cuda() for a in intervals(c))
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        r0, r1, L = int(s["row_off_host"][b]), int(s["row_off_host"][b + 1]), int(s["lens_host"][b])
        if r0 == r1:
            continue
        j = torch.arange(L, device="cuda")
        page = s["page_table"][b, torch.div(j, P, rounding_mode="floor")].long()
        hidden = (j[None] < lo[r0:r1, None]) | (j[None] > hi[r0:r1, None])
        empty = hidden.all(1)
        for h in range(Hkv):
            k, v = s["k_cache"][page, h, j % P].double(), s["v_cache"][page, h, j % P].double()
            for g in range(h * G, h * G + G):
                x = s["q"][r0:r1, g].double() @ k.T / math.sqrt(D)
                if c["softcap"]:
                    x = torch.tanh(x / c["softcap"]) * c["softcap"]
                if s["slopes"] is not None:
                    x = x - s["slopes"][g].double() * (pos[r0:r1, None] - j[None]).abs()
                x[hidden] = -math.inf
                lse[r0:r1, g] = torch.logsumexp(x, 1)
                x[empty] = 0.0
                out[r0:r1, g] = torch.softmax(x, 1) @ v
                out[r0:r1, g][empty] = 0.0
    return {"out": out, "lse": lse}
