"""Rows, slots and page tables of a step, rotary positions with the cache write, and dense attention of new rows, through the C
ABI against plain implementations in 64 bits.

Tolerances.  Whole numbers and copies are exact.  A rotated value is one binary32 expression of two products (each value
within 2^-23 of itself, the sines within 2e-7) rounded once: |err| <= step |value| + 1e-6 (|x| + |y|), step = 2^-11 (f16)
or 2^-8 (bf16).  An attention output is sum p v / sum p with p rounded once to the K/V type and the result once more:
|err| <= step (sum p |v| / sum p) + step |out| + what binary32 sums of scores leave: a score of |s| <= 100 is off by at most
2^-16 and so is the weight, relatively, twice (weight and sum): 4e-5 sum p |v| / sum p.  lse: 2^-16 + 1e-6 |lse|.  Very small
f16 values lose bits below 2^-14: 2^-24 absolute on top.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

D = 128
STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _torch():
    import torch
    assert torch.cuda.is_available()
    return torch


def _absb():
    from paper_2605_12110_amd import absb
    return absb


def _say(msg):
    print(msg, flush=True)


def _layer(Hq=8, Hkv=2, P=16, dt="f16", order="hnd", **kw):
    absb = _absb()
    strides = (Hkv * P * D, P * D, D) if order == "hnd" else (P * Hkv * D, D, Hkv * D)
    strides = kw.pop("kv_strides", strides)
    return absb.Layer(Hq, Hkv, D, P, absb.F16 if dt == "f16" else absb.BF16, None, strides, **kw)


# ------------------------------------------------------------------ rows, slots, page tables
def map_rows_plain(before, after, P, table, ring, cursors, max_rows):
    """One request, one page, one row after the other."""
    table, ring, (head, tail) = table.copy(), None if ring is None else ring.copy(), cursors[:2]
    pages = lambda n: -(-max(n, 0) // P)  # noqa: E731
    off, pos, slot, missing = [0], [], [], 0
    takes = [(b, p) for b in range(len(before)) for p in range(pages(before[b]), pages(after[b]))]
    gives = [(b, p) for b in range(len(before)) for p in range(pages(after[b]), pages(before[b]))]
    if ring is not None:
        missing = max(0, len(takes) - (tail - head)) + sum(p >= table.shape[1] for _, p in takes)
        if not missing:
            given = [table[b, p] for b, p in gives]
            for i, (b, p) in enumerate(takes):
                table[b, p] = ring[(head + i) % len(ring)]
            for i, page in enumerate(given):
                ring[(tail + i) % len(ring)] = page
            head, tail = head + len(takes), tail + len(gives)
    for b in range(len(before)):
        lo = max(before[b], 0)
        for t in range(lo, max(after[b], lo)):
            pos.append(t)
            slot.append(-1 if missing or t // P >= table.shape[1] else int(table[b, t // P]) * P + t % P)
        off.append(len(pos))
    fill = max(0, max_rows - len(pos))
    return off, (pos + [0] * fill)[:max_rows], (slot + [-1] * fill)[:max_rows], table, ring, (head, tail, missing, 0)


def _map_case(before, after, P, width=None, free=None, ring=True, max_rows=None, head=3, seed=0, in_place=True, spare=0):
    torch, absb = _torch(), _absb()
    before, after = np.asarray(before, np.int32), np.asarray(after, np.int32)
    r = np.random.default_rng(seed)
    had, need = -(-np.maximum(before, 0) // P), -(-np.maximum(after, 0) // P)
    width = int(max(had.max(), need.max(), 1)) + spare if width is None else width
    free = int(np.maximum(need - had, 0).sum()) if free is None else free
    n = int(had.sum()) + free
    perm = r.permutation(max(n, 1)).astype(np.int32)
    table = np.full((len(before), width), -77, np.int32)
    at = 0
    for b in range(len(before)):
        k = min(int(had[b]), width)
        table[b, :k] = perm[at:at + k]
        at += int(had[b])
    cap = max(n, 1)
    pages = np.full(cap, -55, np.int32)
    for i in range(free):
        pages[(head + i) % cap] = perm[at + i]
    cursors = np.array([head, head + free, 99, 0], np.int64)
    max_rows = int(np.maximum(after - np.maximum(before, 0), 0).sum()) if max_rows is None else max_rows
    want = map_rows_plain(before.tolist(), after.tolist(), P, table, pages if ring else None, cursors.tolist(), max_rows)
    up = lambda a: torch.from_numpy(a.copy()).cuda()  # noqa: E731
    d_table, d_pages, d_cur, d_after = up(table), up(pages), up(cursors), up(after)
    off = torch.full((len(before) + 1,), -9, dtype=torch.int32, device="cuda")
    # a guard behind the rows: nothing is written there
    pos = torch.full((max_rows + 8,), -9, dtype=torch.int32, device="cuda")
    slot = torch.full((max_rows + 8,), -9, dtype=torch.int64, device="cuda")
    batch = absb.Batch(seq_lens_host=after, seq_lens=d_after, page_table=d_table)
    layer = _layer(P=P)
    out = None if in_place else torch.zeros(4, dtype=torch.int64, device="cuda")
    absb.absb_map_rows(layer, batch, up(before), d_table, off, pos[:max_rows], slot[:max_rows],
                       absb.PageRing(d_pages, d_cur) if ring else None, out)
    torch.cuda.synchronize()
    assert off.tolist() == want[0]
    assert pos[:max_rows].tolist() == want[1] and (pos[max_rows:] == -9).all()
    assert slot[:max_rows].tolist() == want[2] and (slot[max_rows:] == -9).all()
    assert np.array_equal(d_table.cpu().numpy(), want[3])
    if ring:
        assert np.array_equal(d_pages.cpu().numpy(), want[4])
        assert tuple((d_cur if in_place else out).tolist()) == want[5]
        assert in_place or d_cur.tolist() == cursors.tolist()
    return want


def _lens(seed, n, hi, new):
    r = np.random.default_rng(seed)
    before = r.integers(0, hi, n)
    what = r.integers(0, 4, n)
    after = np.where(what == 0, 0, np.where(what == 1, before, np.where(what == 2, before + 1, before + r.integers(0, new, n))))
    return before, after


@pytest.mark.parametrize("before,after,P", [
    ([5], [6], 8),                                     # one request, one token, inside a page
    ([8], [9], 8), ([7], [8], 8),                      # opens a page; fills one
    ([0], [1], 8), ([1], [0], 8), ([0], [0], 8),       # joins, finishes, idle
    ([0, 0, 0], [17, 0, 16], 16),
    ([100, 31, 0, 64], [0, 32, 200, 65], 32),          # gives back and takes in one step
    ([-3, 4], [2, -1], 8),                             # negative lengths count as none
    ([0], [70000], 8),                                 # one long prompt, many work-groups
])
def test_map_rows_by_hand(before, after, P):
    _map_case(before, after, P)
    _map_case(before, after, P, ring=False, width=9000)


@pytest.mark.parametrize("seed,n,hi,new,P", [
    (1, 64, 300, 2, 64), (2, 63, 5000, 300, 16), (3, 1000, 200, 40, 8), (4, 1024, 90, 5, 8), (5, 1025, 90, 5, 8), (6, 2500, 60, 30, 8),
    (7, 5000, 40, 3, 128),
])
def test_map_rows_of_random_steps(seed, n, hi, new, P):
    before, after = _lens(seed, n, hi, new)
    _map_case(before, after, P, seed=seed, in_place=seed % 2 == 0, spare=seed % 3)
    _map_case(before, after, P, seed=seed, ring=False, spare=1)


def test_map_rows_all_or_nothing_when_pages_or_places_are_missing():
    want = _map_case([10, 0, 8], [40, 100, 0], 8, free=3)
    assert want[5][2] > 0 and set(want[2]) == {-1}
    want = _map_case([10, 0], [40, 100], 8, width=6)           # the second table row is too short
    assert want[5][2] == 7
    _map_case([0] * 1500, [9] * 1500, 8, free=2000)            # short by a thousand, found by every work-group
    want = _map_case([0, 5], [20, 9], 8, ring=False, width=2)  # no ring: rows beyond the table have no slot
    assert want[2].count(-1) == 4


def test_map_rows_when_many_pages_come_back():
    _map_case([9000] * 300, [0] * 300, 8)
    _map_case([900] * 2000 + [3], [0] * 2000 + [9], 8, in_place=False)


@pytest.mark.parametrize("before,after,width,missing", [([90, 5], [0, 6], 2, 10), ([90, 5], [20, 30], 2, 11), ([40], [0], 0, 5)])
def test_map_rows_of_tables_too_narrow_for_what_comes_back(before, after, width, missing):
    """Pages of 8: a request shrinks that would hold more of them than its table has entries for.  Nothing changes."""
    torch, absb = _torch(), _absb()
    B = len(before)
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width)
    pages, cursors = torch.arange(100, 120, dtype=torch.int32, device="cuda"), torch.tensor([0, 8, 0, 0], dtype=torch.int64, device="cuda")
    off, pos = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(40, dtype=torch.int32, device="cuda")
    slot = torch.zeros(40, dtype=torch.int64, device="cuda")
    up = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = absb.Batch(seq_lens_host=after, seq_lens=up(after), page_table=table, pt_stride=width)
    absb.absb_map_rows(_layer(P=8), batch, up(before), table, off, pos, slot, absb.PageRing(pages, cursors))
    torch.cuda.synchronize()
    assert cursors.tolist() == [0, 8, missing, 0] and (slot == -1).all()
    assert table.flatten().tolist() == list(range(B * width)) and pages.tolist() == list(range(100, 120))


def test_map_rows_pads_and_cuts_at_max_rows():
    _map_case([3, 0], [9, 30], 8, max_rows=50)
    _map_case([3, 0], [9, 30], 8, max_rows=10)
    _map_case([3, 0], [9, 30], 8, max_rows=0)
    _map_case([3, 0], [9, 30], 8, max_rows=9001)
    _map_case([3] * 1200, [9] * 1200, 8, max_rows=5000)


def test_map_rows_captured_follows_the_lengths_it_finds():
    torch, absb = _torch(), _absb()
    P, n, width = 8, 1100, 12
    r = np.random.default_rng(3)
    cap = n * width
    pages = r.permutation(cap).astype(np.int32)
    table, cursors = np.full((n, width), -1, np.int32), [0, cap, 0, 0]
    lens = np.zeros(n, np.int32)
    d = dict(before=torch.zeros(n, dtype=torch.int32, device="cuda"), after=torch.zeros(n, dtype=torch.int32, device="cuda"),
             table=torch.from_numpy(table.copy()).cuda(), pages=torch.from_numpy(pages.copy()).cuda(),
             cur=torch.tensor(cursors, dtype=torch.int64, device="cuda"))
    M = n * 20
    off = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    pos, slot = torch.zeros(M, dtype=torch.int32, device="cuda"), torch.zeros(M, dtype=torch.int64, device="cuda")
    layer, ring = _layer(P=P), absb.PageRing(d["pages"], d["cur"])
    batch = absb.Batch(seq_lens_host=lens, seq_lens=d["after"], page_table=d["table"])
    call = lambda: absb.absb_map_rows(layer, batch, d["before"], d["table"], off, pos, slot, ring)  # noqa: E731
    call()                                             # nothing grows: a first run outside the graph
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call()
    for step in range(4):
        after = np.minimum(r.integers(0, 20, n) + (lens if step else 0), width * P).astype(np.int32)
        after[r.random(n) < 0.2] = 0
        d["before"].copy_(torch.from_numpy(lens))
        d["after"].copy_(torch.from_numpy(after))
        g.replay()
        torch.cuda.synchronize()
        want = map_rows_plain(lens.tolist(), after.tolist(), P, table, pages, cursors, M)
        assert off.tolist() == want[0] and pos.tolist() == want[1] and slot.tolist() == want[2]
        table, pages, cursors = want[3], want[4], list(want[5])
        assert np.array_equal(d["table"].cpu().numpy(), table) and np.array_equal(d["pages"].cpu().numpy(), pages)
        assert d["cur"].tolist() == cursors and cursors[2] == 0
        lens = after


# ------------------------------------------------------------------ rotary positions
def rotate_plain(x, pos, freq, rot, pairs, amp):
    """x [rows][heads][128] f64; the same in 64 bits, and |x| + |y| of every pair for the tolerance."""
    ang = (pos.astype(np.float64)[:, None] * freq[None])[:, None, :]
    c, s = np.cos(ang), np.sin(ang)
    h = rot // 2
    i0, i1 = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs else (np.arange(h), np.arange(h, rot))
    a, b = x[..., i0], x[..., i1]
    out, size = x.copy(), np.zeros_like(x)
    out[..., i0], out[..., i1] = amp * (a * c - b * s), amp * (a * s + b * c)
    size[..., i0] = size[..., i1] = abs(amp) * (np.abs(a) + np.abs(b))
    return out, size


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("rows,Hq,Hkv,P,rot,pairs,order", [
    (1, 8, 2, 8, 128, False, "hnd"), (1, 32, 8, 64, 128, False, "hnd"), (3, 5, 1, 16, 128, True, "nhd"),
    (17, 40, 8, 64, 64, False, "nhd"), (33, 7, 7, 8, 64, True, "hnd"), (5, 4, 4, 16, 2, False, "hnd"), (5, 4, 2, 16, 2, True, "hnd"),
    (9, 16, 2, 32, 20, False, "nhd"), (9, 6, 2, 32, 22, True, "hnd"), (40, 24, 8, 16, 96, False, "hnd"), (2, 8, 1, 16, 126, False, "hnd"),
    (2100, 3, 1, 64, 112, False, "hnd"), (1300, 32, 8, 16, 128, False, "hnd"), (700, 9, 3, 16, 128, True, "hnd"), (300, 64, 64, 8, 10, False, "nhd"),
])
def test_rotate_store(dt, rows, Hq, Hkv, P, rot, pairs, order):
    torch, absb = _torch(), _absb()
    tdt = torch.float16 if dt == "f16" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(rows * 131 + rot)
    pages = -(-rows // P) + 3
    # one projection's rows, a few elements of something else behind them
    qkv = torch.randn((rows, (Hq + 2 * Hkv) * D + 24), generator=g, device="cuda").to(tdt)
    q, k, v = qkv[:, :-24].view(rows, Hq + 2 * Hkv, D).split((Hq, Hkv, Hkv), 1)
    r = np.random.default_rng(rows)
    pos = r.integers(0, 1 << 21, rows).astype(np.int32)
    pos[0], pos[-1] = 0, 2 ** 31 - 1
    slot = r.permutation(pages * P)[:rows].astype(np.int64)
    slot[r.random(rows) < 0.1] = -1
    amp = 1.25 if rot == 64 else 0.0
    rope = absb.Rope(rot_dim=rot, layout=absb.ROPE_PAIRS if pairs else absb.ROPE_HALVES, base=500000.0, amplitude=amp)
    freq = absb.absb_rope_frequencies(rope)
    kc, vc = (torch.randn((pages, Hkv, P, D) if order == "hnd" else (pages, P, Hkv, D), generator=g, device="cuda").to(tdt) for _ in range(2))
    view = (lambda t: t) if order == "hnd" else (lambda t: t.transpose(1, 2))
    k0, v0 = view(kc).clone(), view(vc).clone()
    q_out = torch.full((rows, Hq, D), float("nan"), dtype=tdt, device="cuda")
    d_pos, d_slot, d_freq = (torch.from_numpy(a).cuda() for a in (pos, slot, freq))
    layer = _layer(Hq, Hkv, P, dt, order)
    before = qkv.clone()
    absb.absb_rotate_store(layer, rope, d_pos, d_slot, d_freq, q, q_out, k, v, kc, vc)
    torch.cuda.synchronize()
    assert torch.equal(qkv.view(torch.int16), before.view(torch.int16))
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    want_q, size_q = rotate_plain(f64(q), pos, freq, rot, pairs, amp or 1.0)
    want_k, size_k = rotate_plain(f64(k), pos, freq, rot, pairs, amp or 1.0)

    def close(got, want, size):
        # angles: exact to 2^-32 turns and position * 2^-52 * |f| on both sides, 2^-19 radians at the farthest position here
        far = np.abs(got - want) - (STEP[dt] * np.abs(want) + 3e-6 * size + 2.0 ** -24)
        assert far.max() <= 0, far.max()
        assert np.array_equal(got[..., rot:], want[..., rot:])

    close(f64(q_out), want_q, size_q)
    used = np.nonzero(slot >= 0)[0]
    d_used = torch.from_numpy(used).cuda()
    page, at = torch.from_numpy(slot[used] // P).cuda(), torch.from_numpy(slot[used] % P).cuda()
    close(f64(view(kc)[page, :, at]), want_k[used], size_k[used])
    assert torch.equal(view(vc)[page, :, at], v[d_used])
    # the rest of the caches is as it was
    for cache, old in ((view(kc).clone(), k0), (view(vc).clone(), v0)):
        cache[page, :, at] = old[page, :, at]
        assert torch.equal(cache.view(torch.int16), old.view(torch.int16))
    # queries alone, in place; keys and values alone
    alone = q.contiguous()
    absb.absb_rotate_store(layer, rope, d_pos, None, d_freq, alone, alone)
    k1, v1 = view(k0.clone()).contiguous(), view(v0.clone()).contiguous()
    absb.absb_rotate_store(layer, rope, d_pos, d_slot, d_freq, k=k, v=v, k_cache=k1, v_cache=v1)
    torch.cuda.synchronize()
    assert torch.equal(alone, q_out) and torch.equal(view(k1), view(kc)) and torch.equal(view(v1), view(vc))


def test_rotate_store_through_rows_behind_the_last():
    """A padded step: rows whose slot is -1 leave the caches alone, whatever their keys hold."""
    torch, absb = _torch(), _absb()
    layer = _layer(4, 2, 8)
    k = torch.full((6, 2, D), float("nan"), dtype=torch.float16, device="cuda")
    kc, vc = torch.zeros((3, 2, 8, D), dtype=torch.float16, device="cuda"), torch.zeros((3, 2, 8, D), dtype=torch.float16, device="cuda")
    rope = absb.Rope()
    freq = torch.from_numpy(absb.absb_rope_frequencies(rope)).cuda()
    absb.absb_rotate_store(layer, rope, torch.zeros(6, dtype=torch.int32, device="cuda"), torch.full((6,), -1, dtype=torch.int64, device="cuda"),
                           freq, k=k, v=k, k_cache=kc, v_cache=vc)
    torch.cuda.synchronize()
    assert not kc.any() and not vc.any()


# ------------------------------------------------------------------ attention of new rows
class Call:
    """A call's inputs, on the device; the same in 64 bits from `plain`."""

    def __init__(self, lens, new, Hq=8, Hkv=2, P=16, dt="f16", order="hnd", shared=None, first=None, seed=0, q_scale=1.5, sm_scale=0.0,
                 softcap=0.0, window=0, slopes=False, prefix=None, docs=None, extra_width=0):
        torch, absb = _torch(), _absb()
        tdt = torch.float16 if dt == "f16" else torch.bfloat16
        self.lens, self.new, self.dt, self.P, self.Hq, self.Hkv = np.asarray(lens, np.int32), np.asarray(new, np.int32), dt, P, Hq, Hkv
        self.softcap, self.window, self.sm_scale = softcap, window, sm_scale or 1 / math.sqrt(D)
        g = torch.Generator(device="cuda").manual_seed(seed)
        B = len(lens)
        n = -(-self.lens.astype(np.int64) // P)
        width = int(n.max()) + extra_width
        table = np.full((B, max(width, 1)), -1, np.int64)
        at = 0
        first = [0, B] if shared is not None and first is None else first
        pre = np.zeros(B, np.int64)
        if shared is not None:
            for j in range(len(shared)):
                m = shared[j] // P
                table[first[j]:first[j + 1], :m] = np.arange(at, at + m)
                pre[first[j]:first[j + 1]] = m
                at += m
        for b in range(B):
            table[b, pre[b]:n[b]] = np.arange(at, at + n[b] - pre[b])
            at += int(n[b] - pre[b])
        pages = at + 1
        perm = np.random.default_rng(seed).permutation(pages)
        table = np.where(table >= 0, perm[np.maximum(table, 0)], 2 ** 30).astype(np.int32)   # (unused entries are never read)
        self.table_host = table
        shape = (pages, Hkv, P, D) if order == "hnd" else (pages, P, Hkv, D)
        mk = lambda: torch.randn(shape, generator=g, device="cuda").to(tdt)  # noqa: E731
        self.k, self.v = mk(), mk()
        self.view = (lambda t: t) if order == "hnd" else (lambda t: t.transpose(1, 2))
        # slots that no token has hold anything
        live = torch.zeros((pages, P), dtype=torch.bool)
        for b in range(B):
            t = np.arange(int(self.lens[b]))
            live[torch.from_numpy(table[b, t // P].astype(np.int64)), torch.from_numpy(t % P)] = True
        dead = ~live.cuda()
        self.view(self.k).transpose(1, 2)[dead] = float("nan")
        self.view(self.v).transpose(1, 2)[dead] = float("inf")
        self.off = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        rows = int(self.off[-1])
        self.rows = rows
        self.q = (q_scale * torch.randn((rows, Hq, D), generator=g, device="cuda")).to(tdt)
        i32 = lambda a: torch.from_numpy(np.asarray(a, np.int32).copy()).cuda()  # noqa: E731
        self.layer = _layer(Hq, Hkv, P, dt, order, sm_scale=sm_scale)
        self.batch = absb.Batch(seq_lens_host=self.lens, seq_lens=i32(self.lens), page_table=i32(table))
        self.r = absb.Rows(self.off, i32(self.off))
        self.shared = None if shared is None else absb.SharedPrefix(first, shared, i32(first), i32(shared))
        self.slopes = np.exp2(-8.0 * np.arange(1, Hq + 1) / Hq).astype(np.float32) if slopes else None
        self.prefix = None if prefix is None else np.asarray(prefix, np.int32)
        self.docs = None if docs is None else np.asarray(docs, np.int32)
        self.opts = absb.ScoreOpts(softcap, window, None if not slopes else torch.from_numpy(self.slopes).cuda(),
                                   None if prefix is None else i32(prefix), None if docs is None else i32(docs))
        self.out = torch.full((rows + 2, Hq, D), float("nan"), dtype=tdt, device="cuda")      # two rows of guard
        self.lse = torch.full((rows + 2, Hq), float("nan"), dtype=torch.float32, device="cuda")
        ws = absb.absb_attend_workspace(self.layer, self.batch, self.r, self.shared)
        self.ws = torch.full((ws + 256,), 0xA5, dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        absb = _absb()
        if self.shared is None:
            absb.absb_attend_rows(self.layer, self.batch, self.r, self.q, self.k, self.v, self.out, self.lse, self.opts, self.ws, stream)
        else:
            absb.absb_attend_shared(self.layer, self.batch, self.r, self.shared, self.q, self.k, self.v, self.out, self.lse, self.opts,
                                    self.ws, stream)

    def intervals(self, b):
        L, n = int(self.lens[b]), int(self.new[b])
        i = np.arange(L - n, L)
        lo, hi = np.zeros(n, np.int64), i.copy()
        if self.prefix is not None:
            hi = np.minimum(np.maximum(hi, self.prefix[b] - 1), L - 1)
        if self.window:
            lo = np.maximum(lo, i - self.window + 1)
        if self.docs is not None:
            lo = np.maximum(lo, self.docs[self.off[b]:self.off[b + 1]])
        return i, lo, hi

    def plain(self):
        """(out, lse, sum p |v| / sum p), in 64 bits, on the device."""
        torch = _torch()
        f = dict(dtype=torch.float64, device="cuda")
        out, mag = torch.zeros((self.rows, self.Hq, D), **f), torch.zeros((self.rows, self.Hq, D), **f)
        lse = torch.full((self.rows, self.Hq), -math.inf, **f)
        G = self.Hq // self.Hkv
        for b in range(len(self.lens)):
            r0, r1, L = int(self.off[b]), int(self.off[b + 1]), int(self.lens[b])
            if r0 == r1:
                continue
            j = np.arange(L)
            page, slot = torch.from_numpy(self.table_host[b, j // self.P].astype(np.int64)).cuda(), torch.from_numpy(j % self.P).cuda()
            i, lo, hi = (torch.from_numpy(a).cuda()[:, None] for a in self.intervals(b))
            jj = torch.from_numpy(j).cuda()[None]
            seen = (jj >= lo) & (jj <= hi)
            for h in range(self.Hq):
                k, v = self.view(self.k)[page, h // G, slot].double(), self.view(self.v)[page, h // G, slot].double()
                x = self.q[r0:r1, h].double() @ k.T.contiguous() * self.sm_scale
                if self.softcap:
                    x = self.softcap * torch.tanh(x / self.softcap)
                if self.slopes is not None:
                    x = x - float(self.slopes[h]) * (i - jj).abs()
                x = x.masked_fill(~seen, -math.inf)
                m = x.amax(1, keepdim=True)
                e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
                s = e.sum(1, keepdim=True)
                ok = s[:, 0] > 0
                out[r0:r1, h][ok], mag[r0:r1, h][ok] = (e @ v / s)[ok], (e @ v.abs() / s)[ok]
                lse[r0:r1, h][ok] = (m + torch.log(s))[ok, 0]
        return out, lse, mag

    def check(self, what=""):
        torch = _torch()
        self.out.fill_(float("nan"))
        self.lse.fill_(float("nan"))
        self.run()
        torch.cuda.synchronize()
        out, lse, mag = self.plain()
        got, got_lse = self.out[:self.rows].double(), self.lse[:self.rows].double()
        assert torch.isnan(self.out[self.rows:]).all() and torch.isnan(self.lse[self.rows:]).all()
        assert torch.isfinite(got).all(), what
        step = STEP[self.dt]
        far = (got - out).abs() - (step * mag + step * out.abs() + 4e-5 * mag + 2.0 ** -24)
        empty = torch.isneginf(lse)
        assert torch.equal(torch.isneginf(got_lse), empty), what
        lse_far = ((got_lse - lse).abs() - (2.0 ** -16 + 1e-6 * lse.abs()))[~empty]
        _say(f"    {what}: max|out - plain| {float((got - out).abs().max()) if self.rows else 0:.2e}, max|lse - plain| "
             f"{float((got_lse - lse).abs()[~empty].max()) if bool((~empty).any()) else 0:.2e}")
        assert not self.rows or float(far.max()) <= 0, what
        assert not lse_far.numel() or float(lse_far.max()) <= 0, what
        assert not got[empty].any(), what


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new,Hq,Hkv,P,order", [
    ([1], [1], 8, 2, 16, "hnd"), ([7], [1], 1, 1, 8, "hnd"), ([64], [1], 4, 4, 64, "nhd"), ([65], [1], 8, 1, 16, "hnd"),
    ([1000], [1], 32, 8, 64, "hnd"), ([5000], [1], 5, 1, 16, "nhd"),
    ([9], [9], 8, 2, 8, "hnd"), ([33], [32], 4, 1, 16, "hnd"), ([128], [128], 6, 2, 32, "nhd"), ([300], [129], 7, 1, 16, "hnd"),
    ([517], [517], 10, 2, 64, "hnd"), ([700], [63], 16, 2, 8, "hnd"),
    ([5, 0, 700, 64, 1], [5, 0, 3, 1, 1], 8, 2, 16, "hnd"), ([40, 900, 2, 333], [0, 0, 0, 300], 12, 4, 16, "nhd"),
    ([100, 200, 300], [0, 0, 0], 8, 2, 16, "hnd"), ([2000] * 9, [1] * 9, 24, 8, 128, "hnd"), ([3000, 17, 900], [4, 1, 2], 8, 1, 64, "hnd"),
])
def test_attend_rows_causal(dt, lens, new, Hq, Hkv, P, order):
    Call(lens, new, Hq, Hkv, P, dt, order, seed=sum(lens)).check(f"{lens} {new} {Hq}/{Hkv} P={P} {dt} {order}")


OPTS = [dict(softcap=30.0), dict(softcap=2000.0), dict(softcap=0.5), dict(window=1), dict(window=100), dict(slopes=True), dict(softcap=20.0, slopes=True, window=333),
        dict(window=2 ** 31 - 1)]


@pytest.mark.parametrize("opts", OPTS, ids=lambda o: "-".join(f"{k}{v}" for k, v in o.items()))
@pytest.mark.parametrize("lens,new,Hq,Hkv,P,dt", [
    ([700, 1, 130], [1, 1, 1], 8, 2, 16, "f16"), ([600, 90, 257], [500, 90, 1], 10, 2, 8, "bf16"), ([4100], [7], 4, 1, 64, "f16"),
])
def test_attend_rows_with_score_options(opts, lens, new, Hq, Hkv, P, dt):
    Call(lens, new, Hq, Hkv, P, dt, seed=5, **opts).check(f"{opts} {lens} {new}")


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("window", [0, 50])
def test_attend_rows_prefix_and_document_masks(slopes, window):
    r = np.random.default_rng(2)
    lens, new = [400, 90, 1, 333], [400, 33, 1, 1]
    docs = np.concatenate([np.sort(r.integers(0, L, n)) for L, n in zip(lens, new)])
    for prefix, doc in (([100, 90, 1, 0], None), (None, docs), ([7, 1000, 0, 333], docs)):
        Call(lens, new, 8, 2, 16, "f16", prefix=prefix, docs=doc, slopes=slopes, window=window).check(f"prefix {prefix} docs {doc is not None}")


def test_attend_rows_that_see_nothing():
    """Documents that start behind the row: alone, whole tiles of them, and all rows of a call."""
    lens, new = [300, 200], [300, 1]
    docs = np.zeros(301, np.int32)
    docs[[0, 5, 63, 299]] = 1000
    docs[128:200] = 2 ** 31 - 1
    docs[300] = 200
    Call(lens, new, 4, 1, 16, "bf16", docs=docs).check("some rows empty")
    Call(lens, new, 4, 1, 16, "f16", docs=np.full(301, 301), window=10).check("all rows empty")
    Call([5000], [2], 4, 1, 16, "f16", docs=[5001, 0]).check("an empty row beside a split one")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new,shared,first,Hq,Hkv,P", [
    ([65, 70], [1, 1], [64], None, 8, 2, 16),
    ([130, 131, 129], [2, 3, 1], [128], None, 4, 1, 64),
    ([64 + 1] * 40, [1] * 40, [64], None, 8, 2, 16),
    ([1000 + i for i in range(9)], [1] * 9, [992], None, 32, 8, 16),
    ([200, 33, 900, 901, 17], [1, 1, 4, 5, 0], [0, 896, 16], [0, 2, 4, 5], 10, 2, 16),
    ([200, 33, 900], [1, 1, 4], [0], None, 10, 2, 16),
    ([2100] * 6, [1] * 6, [2048, 2048, 0], [0, 3, 3, 6], 7, 1, 8),
    ([700, 800], [300, 200], [400], None, 8, 2, 16),
    ([48, 48], [0, 0], [48], None, 8, 2, 16),
])
def test_attend_shared(dt, lens, new, shared, first, Hq, Hkv, P):
    what = f"{lens[:4]} {new[:4]} shared {shared} {dt}"
    Call(lens, new, Hq, Hkv, P, dt, shared=shared, first=first, seed=3).check(what)
    Call(lens, new, Hq, Hkv, P, dt, shared=shared, first=first, seed=4, softcap=10.0, window=150, slopes=True).check(what + " options")


def test_attend_shared_masks():
    docs = np.array([0, 100, 64, 63, 128, 2 ** 31 - 1], np.int32)
    for kw in (dict(docs=docs), dict(prefix=[10, 200, 0]), dict(docs=docs, prefix=[132, 131, 130], window=90)):
        Call([130, 131, 132], [2, 1, 3], 8, 2, 16, "f16", shared=[64], **kw).check(str(kw.keys()))


def test_attend_of_many_requests_and_groups():
    """More owners than a wave looks at in one go: requests, and groups, some of them empty."""
    r = np.random.default_rng(9)
    for B, hi in ((64, 40), (65, 40), (200, 30), (4500, 9)):
        lens = r.integers(0, hi, B)
        Call(lens, np.minimum(lens, r.integers(0, 3, B)), 4, 2, 8, "f16", seed=B).check(f"{B} requests")
    lens = r.integers(9, 30, 300)
    first = np.sort(np.concatenate([[0, 300], r.integers(0, 301, 149)]))
    Call(lens, np.ones(300, np.int64), 4, 2, 8, "f16", shared=(8 * r.integers(0, 2, 150)).tolist(), first=first.tolist(), slopes=True,
         window=20).check("150 groups")
    Call(lens, r.integers(0, 9, 300), 8, 1, 8, "bf16", shared=[0] * 74 + [8] + [0] * 75, first=first.tolist()).check("one group shares")


@pytest.mark.parametrize("Hq,Hkv", [(5, 1), (7, 1), (3, 1), (8, 1), (1, 1)])
def test_attend_windows_over_splits_of_odd_groups(Hq, Hkv):
    for window in (1, 63, 64, 65, 127, 700, 1500):
        Call([9001], [130], Hq, Hkv, 16, "f16", window=window).check(f"chunk, window {window}, {Hq} heads")
        Call([9001, 333], [1, 2], Hq, Hkv, 16, "f16", window=window).check(f"tokens, window {window}, {Hq} heads")


@pytest.mark.parametrize("lens,new,shared", [([50011], [1], None), ([50011], [12], None), ([25000, 26003], [17, 3], None), ([51000, 50500], [5, 4], [50176])])
def test_attend_past_the_caches(lens, new, shared):
    """Contexts of 200 MB, narrow tiles and wide ones, own and shared."""
    Call(lens, new, 32, 8, 64, shared=shared, seed=5).check(f"{lens} {new} {shared}")


@pytest.mark.parametrize("lens,new,Hq,Hkv,opts", [
    ([9100], [1153], 64, 64, dict(window=5000)),                                  # 10 tiles a head, places for 8
    ([9000, 30, 9100, 9050, 9040], [300, 0, 1, 0, 480], 96, 32, dict(window=6011)),   # groups of three across the cut
    ([9000, 8990], [45, 850], 80, 16, dict(softcap=30.0, window=4000)),
    ([30000, 29990], [2600, 2030], 16, 16, dict(slopes=True)),
    ([30000], [1200], 64, 32, dict()),
])
def test_attend_of_equal_tiles_that_fill_the_chip_and_a_bit(lens, new, Hq, Hkv, opts):
    for dt in ("f16", "bf16"):
        c = Call(lens, new, Hq, Hkv, 16, dt, seed=9, **opts)
        n = c.ws.numel() - 256
        c.ws, guard = c.ws[:n], c.ws[n:]
        c.check(f"{lens} {new} {Hq}/{Hkv} {dt} {opts}")
        assert (guard == 0xA5).all()


def test_attend_of_more_than_64_parts():
    absb = _absb()
    c = Call([120001], [1], 8, 1, 64, "f16", shared=[60032])
    assert absb.absb_attend_workspace(c.layer, c.batch, c.r, c.shared) > 64 * 8 * 520
    c.check("prefix and own keys of 60 K")


def test_attend_rows_of_nan_keep_to_themselves():
    torch = _torch()
    for lens, new in (([300], [200]), ([5000], [2]), ([40], [3])):
        c = Call(lens, new)
        c.run()
        torch.cuda.synchronize()
        want, want_lse = c.out[:c.rows].clone(), c.lse[:c.rows].clone()
        c.q[1] = float("nan")
        c.run()
        torch.cuda.synchronize()
        others = [i for i in range(c.rows) if i != 1]
        assert torch.equal(c.out[others], want[others]) and torch.equal(c.lse[others], want_lse[others])
        assert torch.isnan(c.out[1]).all()


def test_attend_without_log_sums():
    torch, absb = _torch(), _absb()
    for c in (Call([600], [200]), Call([9000], [1]), Call([40], [1])):
        c.run()
        torch.cuda.synchronize()
        want = c.out.clone()
        c.out.fill_(0)
        absb.absb_attend_rows(c.layer, c.batch, c.r, c.q, c.k, c.v, c.out, None, c.opts, c.ws)
        torch.cuda.synchronize()
        assert torch.equal(c.out[:c.rows], want[:c.rows])


def test_attend_and_rotate_beyond_4_gib_of_cache():
    """Pages whose offsets pass 32 bits, in bytes and in elements."""
    torch, absb = _torch(), _absb()
    P, Hkv, Hq = 64, 2, 8
    lens, new = [700, 130], [3, 130]
    c = Call(lens, new, Hq, Hkv, P)
    c.run()
    torch.cuda.synchronize()
    want, want_lse = c.out[:c.rows].clone(), c.lse[:c.rows].clone()
    pages = (9 << 30) // (Hkv * P * D * 2)
    K, V = (torch.empty((pages, Hkv, P, D), dtype=torch.float16, device="cuda") for _ in range(2))
    old = c.batch.page_table.clone()
    used = old < c.k.shape[0]
    table = torch.where(used, pages - 1 - old * (pages // (2 * c.k.shape[0])), old).int()
    K[table[used].long()], V[table[used].long()] = c.k[old[used].long()], c.v[old[used].long()]
    c.batch = absb.Batch(seq_lens_host=c.lens, seq_lens=c.batch.seq_lens, page_table=table)
    c.k, c.v = K, V
    c.run()
    torch.cuda.synchronize()
    assert torch.equal(c.out[:c.rows], want) and torch.equal(c.lse[:c.rows], want_lse)
    n = 5
    k, v = (torch.randn((n, Hkv, D), device="cuda").half() for _ in range(2))
    slot = torch.tensor([0, pages * P - 1, pages * P // 2, pages * P // 3, -1], dtype=torch.int64, device="cuda")
    freq = torch.zeros(64, dtype=torch.float64, device="cuda")
    absb.absb_rotate_store(c.layer, absb.Rope(), torch.zeros(n, dtype=torch.int32, device="cuda"), slot, freq, k=k, v=v, k_cache=K, v_cache=V)
    torch.cuda.synchronize()
    page, at = slot[:4] // P, slot[:4] % P
    assert torch.equal(K[page, :, at], k[:4]) and torch.equal(V[page, :, at], v[:4])


def test_attend_of_tokens_half_a_gib_apart():
    """The widest token stride: the last of eight rows is 3.5 GiB behind the first."""
    torch, absb = _torch(), _absb()
    step = 1 << 28
    for n in (1, 8):
        c = Call([8], [n], 4, 1, 8)
        c.run()
        torch.cuda.synchronize()
        want, want_lse = c.out[:c.rows].clone(), c.lse[:c.rows].clone()
        page = int(c.table_host[0, 0])
        K, V = (torch.empty((8 * step,), dtype=torch.float16, device="cuda") for _ in range(2))
        for t in range(8):
            K[t * step:t * step + D], V[t * step:t * step + D] = c.k[page, 0, t], c.v[page, 0, t]
        layer = absb.Layer(4, 1, D, 8, absb.F16, None, (8 * step, D, step))
        batch = absb.Batch(seq_lens_host=c.lens, seq_lens=c.batch.seq_lens, page_table=torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
        absb.absb_attend_rows(layer, batch, c.r, c.q, K, V, c.out, c.lse, None, c.ws)
        torch.cuda.synchronize()
        assert torch.equal(c.out[:c.rows], want) and torch.equal(c.lse[:c.rows], want_lse)


def test_attend_scales_and_out_of_place_widths():
    Call([300], [40], 8, 2, 16, sm_scale=0.5, extra_width=9).check("scale 0.5, wide table")
    Call([300], [1], 8, 2, 16, sm_scale=1e-4).check("scale 1e-4")


def test_attend_output_may_be_the_queries():
    torch, absb = _torch(), _absb()
    for lens, new in (([600], [200]), ([5000], [1])):
        c = Call(lens, new)
        c.run()
        torch.cuda.synchronize()
        want = c.out[:c.rows].clone()
        absb.absb_attend_rows(c.layer, c.batch, c.r, c.q, c.k, c.v, c.q, None, c.opts, c.ws)
        torch.cuda.synchronize()
        assert torch.equal(c.q, want)


def test_attend_is_the_same_every_time_and_in_a_graph():
    torch = _torch()
    for c in (Call([3000, 40], [1, 1]), Call([700, 64], [600, 64], dt="bf16"), Call([1030, 1040, 1100], [1, 1, 2], shared=[1024])):
        c.run()
        torch.cuda.synchronize()
        want, want_lse = c.out.clone(), c.lse.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.run()
        for _ in range(3):
            c.out.fill_(float("nan"))
            c.ws.fill_(0x7f)                     # nothing in the workspace survives
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out[:c.rows], want[:c.rows]) and torch.equal(c.lse[:c.rows], want_lse[:c.rows])


@pytest.mark.parametrize("kw", [dict(lens=[9000, 700, 40, 3], new=[1, 1, 1, 1]), dict(lens=[3000, 2500], new=[70, 200]),
                                dict(lens=[6000, 6000, 5900, 2300], new=[1, 1, 1, 2], shared=[2048], P=32),
                                dict(lens=[6000, 6000], new=[1, 40], window=300)])
def test_a_captured_call_follows_the_lengths_it_finds(kw):
    """Planned for the longest, replayed at shorter ones: a row's context is what the device's lengths say."""
    torch = _torch()
    c = Call(**kw)
    c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        c.run()
    least = np.asarray(kw["new"]) + (kw["shared"][0] if "shared" in kw else 0)
    for step, part in enumerate((0.0, 0.3, 0.8, 1.0)):
        c.lens = (least + (np.asarray(kw["lens"]) - least) * part).astype(np.int32)
        c.batch.seq_lens.copy_(torch.from_numpy(c.lens))
        c.ws.fill_(0x7f)
        c.run = g.replay
        c.check(f"lengths {c.lens.tolist()}")


@pytest.mark.parametrize("lens,new", [([9000], [1]), ([2100, 17, 900], [1, 1, 1]), ([6000] + [100] * 20, [1] * 21), ([3000, 2000], [40, 3])])
def test_attend_workspace_holds_for_every_window(lens, new):
    torch = _torch()
    for window in (0, 1, 17, 63, 64, 100, 129, 500, 1000, 2047, 4096, 100000):
        c = Call(lens, new, window=window)
        n = c.ws.numel() - 256
        c.ws, guard = c.ws[:n], c.ws[n:]
        c.check(f"window {window}")
        assert (guard == 0xA5).all()


def test_the_run_of_a_server():
    """Prompts, then decode steps: rows and pages, rotary positions and cache write, attention of the new rows, the centroid store
    kept current, and the sparse step with a budget that covers the context, which is the attention of single tokens again."""
    torch, absb = _torch(), _absb()
    Hq, Hkv, P, B, steps = 8, 2, 16, 3, 4
    prompt = np.array([70, 5, 133], np.int32)
    cap = prompt + steps
    sizes = [16, 32]
    layer = absb.Layer(Hq, Hkv, D, P, absb.F16, sizes, (Hkv * P * D, P * D, D))
    g = torch.Generator(device="cuda").manual_seed(11)
    pages = int((-(-cap // P)).sum()) + 2
    k, v = (torch.full((pages, Hkv, P, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    width = int((-(-cap // P)).max())
    table = torch.zeros((B, width), dtype=torch.int32, device="cuda")
    ring = absb.PageRing(torch.randperm(pages, generator=g, device="cuda").int(), torch.tensor([0, pages, 0, 0], dtype=torch.int64, device="cuda"))
    before, after = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    rope = absb.Rope(base=10000.0)
    freq_host = absb.absb_rope_frequencies(rope)
    freq = torch.from_numpy(freq_host).cuda()
    batch = absb.Batch(seq_lens_host=prompt, budget_host=cap, seq_lens=after, page_table=table, cap_lens_host=cap,
                       budget=torch.from_numpy(cap).cuda())
    plan = absb.absb_plan(layer, batch)
    batch.cent_off = torch.from_numpy(plan.cent_off).cuda()
    nseg = B * Hkv
    codes = torch.zeros((plan.total_centroids, 64), dtype=torch.uint8, device="cuda")
    qscale, qmin, tail = (torch.zeros((nseg, D), dtype=torch.float32, device="cuda") for _ in range(3))
    ws = torch.zeros(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    have = [[] for _ in range(B)]            # rotated keys, values: 64 bits of what was rounded
    lens = np.zeros(B, np.int32)
    for step in range(1 + steps):
        new = prompt if step == 0 else np.ones(B, np.int32)
        now = lens + new
        rows = int(new.sum())
        after.copy_(torch.from_numpy(now.astype(np.int32)))
        before.copy_(torch.from_numpy(lens.astype(np.int32)))
        batch.seq_lens_host = now.astype(np.int32)
        off = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        pos, slot = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int64, device="cuda")
        absb.absb_map_rows(layer, batch, before, table, off, pos, slot, ring)
        qkv = torch.randn((rows, (Hq + 2 * Hkv), D), generator=g, device="cuda").half()
        q, kn, vn = qkv.split((Hq, Hkv, Hkv), 1)
        qr = torch.empty((rows, Hq, D), dtype=torch.float16, device="cuda")
        absb.absb_rotate_store(layer, rope, pos, slot, freq, q, qr, kn, vn, k, v)
        rec = absb.Rows(np.concatenate([[0], np.cumsum(new)]).astype(np.int32), off)
        out, lse = torch.empty_like(qr), torch.empty((rows, Hq), dtype=torch.float32, device="cuda")
        aw = torch.zeros(absb.absb_attend_workspace(layer, batch, rec), dtype=torch.uint8, device="cuda")
        absb.absb_attend_rows(layer, batch, rec, qr, k, v, out, lse, None, aw)
        torch.cuda.synchronize()
        assert off.tolist() == rec.row_off_host.tolist() and ring.cursors.tolist()[2] == 0
        # in 64 bits, from the projections: one rounding of rotated values (their own test) stands between
        p = pos.cpu().numpy()
        kr = rotate_plain(kn.double().cpu().numpy(), p, freq_host, 128, False, 1.0)[0].astype(np.float16).astype(np.float64)
        qd = rotate_plain(q.double().cpu().numpy(), p, freq_host, 128, False, 1.0)[0].astype(np.float16).astype(np.float64)
        for b in range(B):
            r = slice(int(rec.row_off_host[b]), int(rec.row_off_host[b + 1]))
            have[b] += list(zip(kr[r], vn.double().cpu().numpy()[r]))
            for i, t in zip(range(r.start, r.stop), range(int(lens[b]), int(now[b]))):
                for h in range(Hq):
                    K = np.array([x[0][h // 4] for x in have[b][:t + 1]])
                    V = np.array([x[1][h // 4] for x in have[b][:t + 1]])
                    s = K @ qd[i, h] / math.sqrt(D)
                    w = np.exp(s - s.max())
                    want = w @ V / w.sum()
                    # as in `check`, and a rotated key or query may round the other way on one side: a step of a value, of 128 of
                    # either in a score: 2 sqrt(128) * 2^-11 * |q||k| / sqrt(128) spread over channels, < 0.02 of a weight at the most
                    assert np.abs(out[i, h].double().cpu().numpy() - want).max() <= 2 * STEP["f16"] * np.abs(V).max() + 0.02 * np.abs(V).max()
        if step == 0:
            absb.absb_build_centroids(layer, batch, k, codes, qscale, qmin, ws)
            absb.absb_workspace_init(layer, batch, ws)
            absb.absb_tail_init(layer, batch, k, tail)
        else:
            absb.absb_append_token(layer, batch, k, codes, qscale, qmin, tail)
            sparse, sparse_lse = torch.empty_like(out), torch.empty_like(lse)
            absb.absb_decode_fused(layer, batch, qr, codes, qscale, k, v, sparse, sparse_lse, workspace=ws)
            torch.cuda.synchronize()
            # both round their weights and results once: two steps of values of at most max|v| each
            assert (sparse.double() - out.double()).abs().max() <= 4 * STEP["f16"] * float(vn.abs().max().double().clamp(min=4.0)) * 1.5
            assert (sparse_lse - lse).abs().max() <= 2e-4
        lens = now


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,new,shared,opts", [
    ([700], [600], None, dict()), ([700], [600], None, dict(softcap=50.0)), ([700], [600], None, dict(slopes=True)),   # wide tiles
    ([900], [4], None, dict()), ([9000], [4], None, dict()), ([9000], [300], None, dict(softcap=50.0)),                  # narrow; in parts
    ([1100, 1300], [2, 3], [1024], dict()),
])
def test_attend_outputs_stay_weighted_means(dt, lens, new, shared, opts):
    """The same values at every key: their mean, whatever the weights.  One key in 32 has a score above the others', by 2^0 to 2^8 from
    row to row, so that nearly all of the mass rounds the same way; that must not move the mean.  Sums of n <= 9000 weights in
    binary32, in chains of at most n / 16, are off by n / 16 * 2^-24 < 2^-14 on either side, less than half a step of the values
    (2^-12 and 2^-9, relatively): every output rounds to the value itself."""
    torch = _torch()
    c = Call(lens, new, 8, 2, 16, dt, shared=shared, seed=7, **opts)
    for b, L in enumerate(lens):
        t = np.arange(L)
        page, slot = torch.from_numpy(c.table_host[b, t // 16].astype(np.int64)).cuda(), torch.from_numpy(t % 16).cuda()
        c.view(c.k)[page, :, slot] = torch.from_numpy((t % 32 == 0) * 1.0).cuda().to(c.k.dtype)[:, None, None]
    c.q[:] = torch.linspace(0.05, 0.5, c.rows * c.Hq, device="cuda").view(c.rows, c.Hq, 1).to(c.q.dtype)
    value = (1.0 + torch.arange(D, device="cuda") / 128.0).to(c.v.dtype)
    c.view(c.v)[:] = torch.where(torch.isinf(c.view(c.v)), c.view(c.v), value)
    c.check(f"{lens} {new} {dt} {opts}")
    assert torch.equal(c.out[:c.rows], value.expand(c.rows, c.Hq, D))


@pytest.mark.parametrize("cap", [0.5, 30.0, 50.0, 64.0, 64.5, 100.0, 256.0, 257.0, 2000.0, 1e6])
@pytest.mark.parametrize("lens,new", [([300], [300]), ([3] * 50, [3] * 50)])
def test_attend_caps_are_as_exact_as_they_say(cap, lens, new):
    """Every row sees itself alone, and its score is one product, so that lse is the capped score.  Beside the stated error of the cap
    (3 * 2^-23 cap up to 64, else 2^-19 |x|), the angle's two factors and its product, the result's factor and product
    are off by 2^-24 each: 2^-21 |x|, and 2^-149 where nothing is left to be relative to."""
    torch = _torch()
    c = Call(lens, new, 8, 2, 16, "f16", softcap=cap, window=1, seed=3)
    c.k[..., 1:] = torch.where(torch.isnan(c.k[..., 1:]), c.k[..., 1:], 0.0)
    # arguments of tanh: 0.25 either way, most of them, up to a few; with sqrt(128) for the scale
    y = torch.linspace(-1.2, 1.2, c.rows * c.Hq, device="cuda", dtype=torch.float64)
    y = torch.where(torch.arange(len(y), device="cuda") % 3 == 0, y * 3, y * 0.4).view(c.rows, c.Hq)
    most = min(60000.0, 40 * cap)
    c.q[:, :, 0] = (y / 4 * most).to(c.q.dtype)
    c.k[..., 0] = torch.where(torch.isnan(c.k[..., 0]), c.k[..., 0], cap * math.sqrt(D) * 4 / most).to(c.k.dtype)
    c.run()
    torch.cuda.synchronize()
    x = c.plain()[1]
    assert (x.abs() > 0.9 * cap).any() and (x.abs() < 0.1 * cap).any()
    far = (c.lse[:c.rows].double() - x).abs() - ((3 * 2.0 ** -23 * cap if cap <= 64 else 2.0 ** -19 * x.abs()) + 2.0 ** -21 * x.abs() + 2.0 ** -149)
    _say(f"    cap {cap} {new[:2]}: max|lse - plain| {float((c.lse[:c.rows].double() - x).abs().max()):.2e}, of it beyond {float(far.max()):.2e}")
    assert float(far.max()) <= 0


@pytest.mark.parametrize("B,at", [(63, (0, 30, 62)), (64, (0, 31, 63)), (90, (89,)), (300, (0,)), (300, (7, 150, 151)), (400, (399,))])
@pytest.mark.parametrize("opts", [dict(), dict(window=20000)])
def test_attend_of_a_tail_among_idle_requests(B, at, opts):
    """Equal tiles that fill the chip and a bit, brought by a few of many requests: which tiles are cut, and whose parts are merged,
    goes by slots, of which idle requests have one each."""
    lens, new = np.zeros(B, np.int64), np.zeros(B, np.int64)
    for i, b in enumerate(at):
        new[b] = 1050 // len(at) + i
        lens[b] = 30000 - 7 * i
    for dt in ("f16", "bf16"):
        c = Call(lens, new, 64, 8, 16, dt, seed=B, **opts)                   # 66 tiles a head, places for 64
        # (partial results of some rows only)
        assert 0 < _absb().absb_attend_workspace(c.layer, c.batch, c.r, None, c.opts) < c.rows * 64 * 524
        n = c.ws.numel() - 256
        c.ws, guard = c.ws[:n], c.ws[n:]
        c.check(f"{B} requests, rows of {at} {dt} {opts}")
        assert (guard == 0xA5).all()


@pytest.mark.parametrize("rot,pairs", [(128, False), (128, True), (64, False), (22, True)])
def test_rotate_angles_are_as_exact_as_they_say(rot, pairs):
    """Pairs that all but cancel, 256 (sin a, cos a) in f16 at angle a: x cos a - y sin a is what the rounding of x and y leaves, so that
    its own rounding hides little.  Angle: 2^-25 turns = 1.9e-7, and position * 2^-52 |f|; hardware sine 1.3e-7; two factors,
    two products and a sum in binary32: 4 * 2^-24 = 2.4e-7; the oracle's own product 2^-53 position |f|."""
    torch, absb = _torch(), _absb()
    pos = np.concatenate([np.arange(64), 2 ** np.arange(6, 31), 2 ** np.arange(7, 32) - 1, np.random.default_rng(1).integers(0, 1 << 20, 100)])
    pos = pos.astype(np.int32)
    n, half = len(pos), rot // 2
    rope = absb.Rope(rot_dim=rot, layout=absb.ROPE_PAIRS if pairs else absb.ROPE_HALVES, base=10000.0)
    freq = absb.absb_rope_frequencies(rope)
    i0, i1 = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if pairs else (np.arange(half), np.arange(half, rot))
    x = np.random.default_rng(2).standard_normal((n, 1, D))
    angle = pos[:, None].astype(np.float64) * freq[None]
    x[:, 0, i0], x[:, 0, i1] = 256 * np.sin(angle), 256 * np.cos(angle)
    q = torch.from_numpy(x).half().cuda()
    out = torch.empty_like(q)
    absb.absb_rotate_store(_layer(1, 1), rope, torch.from_numpy(pos).cuda(), None, torch.from_numpy(freq).cuda(), q, out)
    torch.cuda.synchronize()
    want, size = rotate_plain(q.double().cpu().numpy(), pos, freq, rot, pairs, 1.0)
    far = np.zeros((n, 1, D))
    far[:, 0, i0] = far[:, 0, i1] = 1.9e-7 + 1.3e-7 + 2.4e-7 + pos[:, None] * 2.0 ** -51 * freq[None]
    err = np.abs(out.double().cpu().numpy() - want)
    _say(f"    rot {rot}: {float(((err - STEP['f16'] * np.abs(want) - 2.0 ** -24) / np.maximum(size, 1e-9))[:, :, i0].max()):.2e} of |x| + |y|")
    assert (err <= far * size + STEP["f16"] * np.abs(want) + 2.0 ** -24).all()


def test_the_run_of_a_server_with_a_shared_prefix():
    """Requests on a common prefix join, grow, finish and are replaced; their own pages go through the ring, the prefix's are taken
    and given back by a call for the prefix alone.  Every page is with one owner at any time."""
    torch, absb = _torch(), _absb()
    Hq, Hkv, P, S, B, pages = 8, 2, 16, 48, 4, 24
    g = torch.Generator(device="cuda").manual_seed(21)
    layer = _layer(Hq, Hkv, P)
    k, v = (torch.full((pages, Hkv, P, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    ring = absb.PageRing(torch.randperm(pages, generator=g, device="cuda").int(), torch.tensor([0, pages, 0, 0], dtype=torch.int64, device="cuda"))
    rope, freq = absb.Rope(), torch.zeros(64, dtype=torch.float64, device="cuda")       # (no turn: keys are stored as they are)
    up = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731

    def step(table, before, after):
        """Rows and pages, new keys and values into the cache; what `absb_attend_shared` takes."""
        new = [max(a - b, 0) for b, a in zip(before, after)]
        rows = sum(new)
        off, pos, slot = up([0] * (len(new) + 1)), up([0] * rows), torch.zeros(rows, dtype=torch.int64, device="cuda")
        batch = absb.Batch(seq_lens_host=after, seq_lens=up(after), page_table=table)
        absb.absb_map_rows(layer, batch, up(before), table, off, pos, slot, ring)
        qkv = torch.randn((rows, Hq + 2 * Hkv, D), generator=g, device="cuda").half()
        q, kn, vn = qkv.split((Hq, Hkv, Hkv), 1)
        absb.absb_rotate_store(layer, rope, pos, slot, freq, k=kn, v=vn, k_cache=k, v_cache=v)
        rec = absb.Rows(np.concatenate([[0], np.cumsum(new)]).astype(np.int32), off)
        assert off.tolist() == rec.row_off_host.tolist() and ring.cursors.tolist()[2] == 0
        return batch, rec, q.contiguous(), kn.double(), vn.double()

    prefix = torch.full((1, S // P), -1, dtype=torch.int32, device="cuda")
    _, _, _, pk, pv = step(prefix, [0], [S])
    table = torch.full((B, 8), -1, dtype=torch.int32, device="cuda")
    shared = absb.SharedPrefix([0, B], [S], up([0, B]), up([S]))
    table[:, :S // P] = prefix
    have = [(pk, pv)] * B
    lens = [S] * B
    for after in ([S + 5, S + 20, S, S + 1], [S + 6, S, S + 17, S + 2], [S + 7, S, S + 18, S + 40], [S + 8, S + 33, S, S], [S, S + 34, S + 16, S + 1]):
        batch, rec, q, kn, vn = step(table, lens, after)
        # every page: free, the prefix's, or one request's
        head, tail = ring.cursors.tolist()[:2]
        free = [int(ring.pages[i % pages]) for i in range(head, tail)]
        held = [int(x) for b in range(B) for x in table[b, S // P:-(-after[b] // P)]]
        assert sorted(free + held + prefix[0].tolist()) == list(range(pages))
        out = torch.empty_like(q)
        lse = torch.empty((len(q), Hq), dtype=torch.float32, device="cuda")
        ws = torch.zeros(absb.absb_attend_workspace(layer, batch, rec, shared), dtype=torch.uint8, device="cuda")
        absb.absb_attend_shared(layer, batch, rec, shared, q, k, v, out, lse, None, ws)
        torch.cuda.synchronize()
        off = rec.row_off_host
        for b in range(B):
            r = slice(int(off[b]), int(off[b + 1]))
            K, V = (torch.cat([old, new[r]]) if after[b] > lens[b] else old[:after[b]] for old, new in zip(have[b], (kn, vn)))
            have[b] = (K, V)
            for i in range(r.start, r.stop):
                n = after[b] - (r.stop - 1 - i)
                for h in range(Hq):
                    s = (K[:n, h // 4] * q[i, h].double()).sum(1) / math.sqrt(D)
                    w = torch.softmax(s, 0)[:, None]
                    want, mag = (w * V[:n, h // 4]).sum(0), (w * V[:n, h // 4].abs()).sum(0)
                    far = (out[i, h].double() - want).abs() - (STEP["f16"] * (mag + want.abs()) + 4e-5 * mag + 2.0 ** -24)
                    assert float(far.max()) <= 0 and abs(float(lse[i, h]) - float(torch.logsumexp(s, 0))) <= 2.0 ** -16 + 1e-6 * float(s.abs().max())
        lens = after
    step(table, lens, [S] * B)
    step(prefix, [S], [0])
    head, tail = ring.cursors.tolist()[:2]
    assert sorted(int(ring.pages[i % pages]) for i in range(head, tail)) == list(range(pages))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("rot,pairs", [(128, False), (64, False), (128, True), (40, True), (20, False)])
@pytest.mark.parametrize("rows", [6007, 13001])
def test_rotate_of_more_than_caches_keep(dt, rot, pairs, rows):
    """70 and 152 MB of 48 heads, which pass the caches by on the way in, and out: the same bits as in stretches of 1000 rows."""
    torch, absb = _torch(), _absb()
    Hq, Hkv, P = 32, 8, 16
    tdt = torch.float16 if dt == "f16" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(rows + rot)
    qkv = torch.randn((rows, (Hq + 2 * Hkv), D), generator=g, device="cuda").to(tdt)
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    pages = rows // P + 2
    slot = torch.randperm(pages * P, generator=g, device="cuda")[:rows]
    slot[::97] = -1
    pos = torch.randint(0, 1 << 20, (rows,), generator=g, device="cuda", dtype=torch.int32)
    rope = absb.Rope(rot_dim=rot, layout=absb.ROPE_PAIRS if pairs else absb.ROPE_HALVES, base=500000.0)
    freq = torch.from_numpy(absb.absb_rope_frequencies(rope)).cuda()
    layer = _layer(Hq, Hkv, P, dt)
    got, want = ([torch.full((rows, Hq, D), float("nan"), dtype=tdt, device="cuda")] +
                 [torch.zeros((pages, Hkv, P, D), dtype=tdt, device="cuda") for _ in range(2)] for _ in range(2))
    absb.absb_rotate_store(layer, rope, pos, slot, freq, q, got[0], k, v, got[1], got[2])
    for a in range(0, rows, 1000):
        b = min(a + 1000, rows)
        absb.absb_rotate_store(layer, rope, pos[a:b], slot[a:b], freq, q[a:b], want[0][a:b], k[a:b], v[a:b], want[1], want[2])
    torch.cuda.synchronize()
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(got, want))
    alone = q.contiguous()        # queries alone, in place
    absb.absb_rotate_store(layer, rope, pos, None, freq, alone, alone)
    torch.cuda.synchronize()
    assert torch.equal(alone.view(torch.int16), got[0].view(torch.int16))


@pytest.mark.parametrize("lens,new", [([700], [600]), ([4000], [4])])
def test_attend_of_weights_below_the_normal_values_of_f16(lens, new):
    """As above, with one key in 256 whose weight is 1 and the others' 2^-14 to 2^-18: products and sums both keep them."""
    torch = _torch()
    c = Call(lens, new, 8, 2, 16, "f16", seed=7)
    t = np.arange(lens[0])
    page, slot = torch.from_numpy(c.table_host[0, t // 16].astype(np.int64)).cuda(), torch.from_numpy(t % 16).cuda()
    c.view(c.k)[page, :, slot] = torch.from_numpy((t % 256 == 0) * 1.0).cuda().half()[:, None, None]
    c.q[:] = torch.linspace(14 / 16.32, 18 / 16.32, c.rows * c.Hq, device="cuda").view(c.rows, c.Hq, 1).half()   # sqrt(128) log2(e) = 16.32
    value = (1.0 + torch.arange(D, device="cuda") / 128.0).half()
    c.view(c.v)[:] = torch.where(torch.isinf(c.view(c.v)), c.view(c.v), value)
    c.check(f"{lens} {new}")
    assert torch.equal(c.out[:c.rows], value.expand(c.rows, c.Hq, D))
