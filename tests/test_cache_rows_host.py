"""Host side of the entry points around the cache (no GPU): frequencies of rotary positions against their formulas, workspace sizes,
and what is refused before anything is enqueued.  Addresses here are never followed: every call is refused, or has
nothing to do."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from paper_2605_12110_amd import absb

D, AT = 128, 1 << 20      # AT: a 16-byte aligned address that nobody follows


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(absb.LIB_PATH):
        from paper_2605_12110_amd.build import build_library
        build_library(force=False)


def _layer(**kw):
    d = dict(num_q_heads=32, num_kv_heads=8, head_dim=D, page_size=64, dtype=absb.F16, block_size=None,
             kv_strides=(8 * 64 * D, 64 * D, D))
    d.update(kw)
    return absb.Layer(**d)


def _batch(lens, width=None, P=64):
    return absb.Batch(seq_lens_host=list(lens), seq_lens=AT, page_table=AT, pt_stride=(max(lens) + P - 1) // P if width is None else width)


def _rows(new):
    return absb.Rows(np.concatenate([[0], np.cumsum(new)]).astype(np.int32), AT)


def _refused(status, f, *a, **kw):
    with pytest.raises(absb.AbsbError) as e:
        f(*a, stream=0, **kw)
    assert e.value.status == status, e.value


# ------------------------------------------------------------------ frequencies
@pytest.mark.parametrize("R", [2, 4, 64, 96, 126, 128])
def test_frequencies_plain_linear_and_base(R):
    i = np.arange(R // 2)
    f = absb.absb_rope_frequencies(absb.Rope(rot_dim=R, base=500000.0))
    assert np.allclose(f, 500000.0 ** (-2.0 * i / R), rtol=1e-14) and f[0] == 1.0
    lin = absb.absb_rope_frequencies(absb.Rope(rot_dim=R, base=500000.0, scaling=absb.ROPE_LINEAR, factor=8.0))
    assert np.allclose(lin, f / 8.0, rtol=1e-14)
    if R > 2:      # the lowest frequency is divided by the factor, the highest stays
        b = absb.absb_rope_frequencies(absb.Rope(rot_dim=R, base=500000.0, scaling=absb.ROPE_BASE, factor=8.0))
        assert b[0] == 1.0 and math.isclose(b[-1], f[-1] / 8.0, rel_tol=1e-12) and (np.diff(b) < 0).all()


def test_frequencies_by_turns():
    rope = absb.Rope(rot_dim=128, base=500000.0, scaling=absb.ROPE_BY_TURNS, factor=8.0, original_len=8192.0, low_turns=1.0, high_turns=4.0)
    f0, f = absb.absb_rope_frequencies(absb.Rope(base=500000.0)), absb.absb_rope_frequencies(rope)
    turns = 8192.0 * f0 / (2 * math.pi)
    assert (turns > 4).any() and (turns < 1).any() and ((turns > 1) & (turns < 4)).any()
    for t, a, b in zip(turns, f0, f):
        keep = min(1.0, max(0.0, (t - 1.0) / 3.0))
        assert math.isclose(b, a * keep + a / 8.0 * (1 - keep), rel_tol=1e-13)
    assert np.array_equal(f[turns >= 4], f0[turns >= 4])


@pytest.mark.parametrize("kw,status", [
    (dict(rot_dim=0), absb.ERR_BAD_SHAPE), (dict(rot_dim=3), absb.ERR_BAD_SHAPE), (dict(rot_dim=130), absb.ERR_BAD_SHAPE),
    (dict(layout=2), absb.ERR_UNSUPPORTED), (dict(scaling=4), absb.ERR_UNSUPPORTED), (dict(scaling=-1), absb.ERR_UNSUPPORTED),
    (dict(base=1.0), absb.ERR_BAD_SHAPE), (dict(base=math.nan), absb.ERR_BAD_SHAPE), (dict(base=math.inf), absb.ERR_BAD_SHAPE),
    (dict(scaling=1, factor=0.5), absb.ERR_BAD_SHAPE), (dict(scaling=1, factor=math.nan), absb.ERR_BAD_SHAPE),
    (dict(scaling=2, factor=2.0, rot_dim=2), absb.ERR_BAD_SHAPE), (dict(amplitude=math.nan), absb.ERR_BAD_SHAPE),
    (dict(scaling=3, factor=2.0, original_len=0.0, low_turns=1.0, high_turns=4.0), absb.ERR_BAD_SHAPE),
    (dict(scaling=3, factor=2.0, original_len=99.0, low_turns=4.0, high_turns=4.0), absb.ERR_BAD_SHAPE),
    (dict(scaling=3, factor=2.0, original_len=99.0, low_turns=-1.0, high_turns=4.0), absb.ERR_BAD_SHAPE),
])
def test_frequencies_refusals(kw, status):
    with pytest.raises(absb.AbsbError) as e:
        absb.absb_rope_frequencies(absb.Rope(**kw))
    assert e.value.status == status


# ------------------------------------------------------------------ refusals
class _T:
    """Stands for a dense device tensor of whole rows."""

    def __init__(self, *shape, at=AT, stride0=None, size=2):
        self.shape, self._at, self._s0, self._size = shape, at, stride0, size

    def data_ptr(self):
        return self._at

    def numel(self):
        return math.prod(self.shape)

    def element_size(self):
        return self._size

    def stride(self):
        dense = tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))
        return dense if self._s0 is None else (self._s0, *dense[1:])

    def is_contiguous(self):
        return self._s0 is None


def _map(layer=None, batch=None, before=AT, table=AT, off=AT, pos=None, slot=None, ring=None, **kw):
    return (layer or _layer(), batch or _batch([5]), before, table, off, pos or _T(4), slot or _T(4), ring)


def test_map_rows_refusals():
    f = absb.absb_map_rows
    _refused(absb.ERR_BAD_SHAPE, f, *_map(layer=_layer(page_size=12)))
    _refused(absb.ERR_NULL, f, *_map(before=None))
    _refused(absb.ERR_NULL, f, *_map(table=None))
    _refused(absb.ERR_NULL, f, *_map(off=None))
    _refused(absb.ERR_NULL, f, *_map(pos=_T(4, at=None)))
    _refused(absb.ERR_BAD_SHAPE, f, *_map(pos=_T(5)))
    _refused(absb.ERR_BAD_SHAPE, f, *_map(pos=_T((1 << 30) + 1), slot=_T((1 << 30) + 1)))
    _refused(absb.ERR_NULL, f, *_map(batch=absb.Batch(seq_lens_host=[5], pt_stride=1)))
    _refused(absb.ERR_BAD_SHAPE, f, *_map(batch=_batch([1] * 65536)))
    _refused(absb.ERR_BAD_SHAPE, f, *_map(batch=_batch([5], width=-1)))
    _refused(absb.ERR_BAD_SHAPE, f, *_map(ring=absb.PageRing(_T(0), _T(4))))
    _refused(absb.ERR_NULL, f, *_map(ring=absb.PageRing(_T(9), _T(4, at=None))))
    lib = absb.load()
    assert lib.absb_map_rows(None, None, None, None, None, 0, None, None, None, None) == absb.ERR_NULL


def _rot(n=3, **kw):
    d = dict(layer=_layer(), rope=absb.Rope(), row_pos=_T(n), row_slot=_T(n), freq=AT, q=_T(n, 32, D), q_out=_T(n, 32, D, at=AT + 4096),
             k=_T(n, 8, D), v=_T(n, 8, D), k_cache=AT, v_cache=AT)
    d.update(kw)
    return d


@pytest.mark.parametrize("kw,status", [
    (dict(layer=_layer(head_dim=64)), absb.ERR_UNSUPPORTED), (dict(layer=_layer(num_q_heads=72), q=_T(3, 72, D), q_out=_T(3, 72, D)), absb.ERR_UNSUPPORTED),
    (dict(layer=_layer(dtype=3)), absb.ERR_UNSUPPORTED), (dict(layer=_layer(kv_strides=(4, 4, 4))), absb.ERR_BAD_SHAPE),
    (dict(layer=_layer(kv_strides=(8 * 64 * D, 64 * D, (1 << 28) + 8))), absb.ERR_UNSUPPORTED),
    (dict(rope=absb.Rope(rot_dim=7)), absb.ERR_BAD_SHAPE), (dict(row_pos=_T(3, at=None)), absb.ERR_NULL), (dict(row_slot=None), absb.ERR_NULL),
    (dict(freq=None), absb.ERR_NULL), (dict(q=None), absb.ERR_NULL), (dict(q_out=None), absb.ERR_NULL), (dict(k=None), absb.ERR_NULL),
    (dict(v=None), absb.ERR_NULL), (dict(k_cache=None), absb.ERR_NULL), (dict(v_cache=None), absb.ERR_NULL),
    (dict(q=None, q_out=None, k=None, v=None), absb.ERR_NULL),
    (dict(q=_T(3, 32, D, stride0=32 * D + 4)), absb.ERR_BAD_SHAPE), (dict(k=_T(3, 8, D, stride0=8 * D - 8)), absb.ERR_BAD_SHAPE),
    (dict(v=_T(3, 8, D, stride0=8 * D + 1)), absb.ERR_BAD_SHAPE), (dict(q=_T(3, 32, D, at=AT + 8)), absb.ERR_BAD_SHAPE),
    (dict(k_cache=AT + 2), absb.ERR_BAD_SHAPE), (dict(q=_T(3, 32, D, at=AT + 4096, stride0=48 * D)), absb.ERR_BAD_SHAPE),     # in place, rows apart
    (dict(q=_T(4, 32, D)), absb.ERR_BAD_SHAPE), (dict(q=_T(3, 31, D)), absb.ERR_BAD_SHAPE), (dict(q_out=_T(3, 32, D, stride0=8192)), absb.ERR_BAD_SHAPE),
])
def test_rotate_store_refusals(kw, status):
    _refused(status, absb.absb_rotate_store, **_rot(**kw))


def test_rotate_store_of_no_rows_does_nothing():
    absb.absb_rotate_store(stream=0, **_rot(n=0))


def _att(lens=(100, 200), new=(1, 2), layer=None, batch=None, rows=None, q=AT, k=AT, v=AT, out=AT, opts=None, ws=None, **kw):
    return (layer or _layer(), batch or _batch(lens), rows or _rows(new), q, k, v, out, None, opts, ws)


BIG_WS = _T(1 << 40, size=1)


@pytest.mark.parametrize("kw,status", [
    (dict(layer=_layer(head_dim=64)), absb.ERR_UNSUPPORTED), (dict(layer=_layer(num_q_heads=33)), absb.ERR_BAD_SHAPE),
    (dict(layer=_layer(num_q_heads=72)), absb.ERR_UNSUPPORTED), (dict(layer=_layer(sm_scale=-1.0)), absb.ERR_BAD_SHAPE),
    (dict(layer=_layer(page_size=4)), absb.ERR_BAD_SHAPE), (dict(layer=_layer(kv_strides=(8, 8, (1 << 28) + 8))), absb.ERR_UNSUPPORTED),
    (dict(new=(101, 1)), absb.ERR_BAD_SHAPE), (dict(lens=(0, 5), new=(1, 1)), absb.ERR_BAD_SHAPE), (dict(lens=(-1, 5), new=(0, 1)), absb.ERR_BAD_SHAPE),
    (dict(rows=absb.Rows([1, 2, 3], AT)), absb.ERR_BAD_SHAPE), (dict(rows=absb.Rows([0, 2, 1], AT)), absb.ERR_BAD_SHAPE),
    (dict(rows=absb.Rows(None, AT)), absb.ERR_NULL), (dict(rows=absb.Rows([0, 1, 2], None)), absb.ERR_NULL),
    (dict(batch=_batch((100, 200), width=3)), absb.ERR_BAD_SHAPE),
    (dict(q=None), absb.ERR_NULL), (dict(k=None), absb.ERR_NULL), (dict(v=None), absb.ERR_NULL), (dict(out=None), absb.ERR_NULL),
    (dict(q=AT + 8), absb.ERR_BAD_SHAPE), (dict(out=AT + 2), absb.ERR_BAD_SHAPE), (dict(k=AT + 4), absb.ERR_BAD_SHAPE),
    (dict(opts=absb.ScoreOpts(softcap=-1.0)), absb.ERR_BAD_SHAPE), (dict(opts=absb.ScoreOpts(softcap=math.nan)), absb.ERR_BAD_SHAPE),
    (dict(opts=absb.ScoreOpts(softcap=math.inf)), absb.ERR_BAD_SHAPE), (dict(opts=absb.ScoreOpts(softcap=1e-31)), absb.ERR_BAD_SHAPE),
    (dict(opts=absb.ScoreOpts(softcap=1e31)), absb.ERR_BAD_SHAPE), (dict(q=_T(3, 32, D, stride0=48 * D)), absb.ERR_BAD_SHAPE),
    (dict(out=_T(3, 32, D, stride0=48 * D)), absb.ERR_BAD_SHAPE), (dict(lens=(100, (1 << 30) + 1)), absb.ERR_BAD_SHAPE),
    (dict(lens=(1 << 27, 5), new=(1 << 27, 1)), absb.ERR_BAD_SHAPE),          # 2^32 pairs of row and head
    (dict(opts=absb.ScoreOpts(window=-1)), absb.ERR_BAD_SHAPE),
    (dict(lens=(5000, 9000)), absb.ERR_WORKSPACE), (dict(lens=(5000, 9000), ws=_T(100, size=1)), absb.ERR_WORKSPACE),
    (dict(lens=(5000, 9000), ws=_T(1 << 40, at=AT + 16, size=1)), absb.ERR_WORKSPACE),
])
def test_attend_rows_refusals(kw, status):
    _refused(status, absb.absb_attend_rows, *_att(**kw))


@pytest.mark.parametrize("shared,status", [
    (absb.SharedPrefix([0, 2], [65], AT, AT), absb.ERR_BAD_SHAPE),            # not whole pages
    (absb.SharedPrefix([0, 2], [-64], AT, AT), absb.ERR_BAD_SHAPE),
    (absb.SharedPrefix([0, 2], [128], AT, AT), absb.ERR_BAD_SHAPE),           # longer than the first request's older tokens
    (absb.SharedPrefix([0, 1], [64], AT, AT), absb.ERR_BAD_SHAPE),            # a request without a group
    (absb.SharedPrefix([1, 2], [64], AT, AT), absb.ERR_BAD_SHAPE),
    (absb.SharedPrefix([0, 2, 1, 2], [0, 0, 0], AT, AT), absb.ERR_BAD_SHAPE),
    (absb.SharedPrefix([0, 3, 2], [0, 0], AT, AT), absb.ERR_BAD_SHAPE),
    (absb.SharedPrefix([0, 2], [64], None, AT), absb.ERR_NULL), (absb.SharedPrefix([0, 2], [64], AT, None), absb.ERR_NULL),
])
def test_attend_shared_refusals(shared, status):
    layer, batch, rows, q, k, v, out, lse, opts, _ = _att()
    _refused(status, absb.absb_attend_shared, layer, batch, rows, shared, q, k, v, out, lse, opts, BIG_WS)


def test_attend_refuses_null_records():
    lib = absb.load()
    cl, cb, cr = _layer().c(), _batch([5]).c(), _rows([1]).c()
    n = C.c_size_t(0)
    assert lib.absb_attend_workspace(None, C.byref(cb), C.byref(cr), None, None, C.byref(n)) == absb.ERR_NULL
    assert lib.absb_attend_workspace(C.byref(cl), None, C.byref(cr), None, None, C.byref(n)) == absb.ERR_NULL
    assert lib.absb_attend_workspace(C.byref(cl), C.byref(cb), None, None, None, C.byref(n)) == absb.ERR_NULL
    assert lib.absb_attend_workspace(C.byref(cl), C.byref(cb), C.byref(cr), None, None, None) == absb.ERR_NULL
    assert lib.absb_attend_shared(C.byref(cl), C.byref(cb), C.byref(cr), None, AT, AT, AT, AT, None, None, None, 0, None) == absb.ERR_NULL


def test_what_a_launch_or_a_tensor_cannot_hold_is_refused():
    _refused(absb.ERR_BAD_SHAPE, absb.absb_rotate_store, **_rot(n=1 << 26))
    _refused(absb.ERR_BAD_SHAPE, absb.absb_rotate_store, **_rot(row_slot=_T(2)))
    _refused(absb.ERR_BAD_SHAPE, absb.absb_attend_rows, *_att(lens=(1 << 25, 1), new=(1 << 25, 0), ws=BIG_WS))   # 2^30 pairs of row and head
    for kw in (dict(q=_T(2, 32, D)), dict(out=_T(3, 31, D))):
        _refused(absb.ERR_BAD_SHAPE, absb.absb_attend_rows, *_att(**kw))
    # many requests of which one is long: cut no further than a launch has room for, and refused if it never had
    n, layer = 65535, _layer(num_q_heads=64, num_kv_heads=64)
    lens = np.full(n, 64, np.int32)
    lens[0] = 1 << 30
    batch, rows = absb.Batch(seq_lens_host=lens, seq_lens=AT, page_table=AT, pt_stride=1 << 24), _rows(np.ones(n, np.int32))
    parts = absb.absb_attend_workspace(layer, batch, rows, None, absb.ScoreOpts()) // (n * 64 * 520)
    assert parts <= 3             # 65535 + 65535 / 32 slots of 64 heads are a quarter of the work-groups of a launch


def test_attend_of_no_rows_does_nothing():
    absb.absb_attend_rows(*_att(new=(0, 0)), stream=0)
    absb.absb_attend_rows(*_att(lens=(0, 0), new=(0, 0), q=None, out=None), stream=0)


# ------------------------------------------------------------------ workspaces
@pytest.mark.parametrize("lens,new", [([131072], [1]), ([4096], [4096]), ([9000, 17, 4000], [1, 1, 1]), ([131072] + [100] * 63, [1] * 64),
                                      ([2048], [1]), ([30000, 30000], [40, 3])])
def test_workspace_sizes(lens, new):
    # at most 65 parts a row and query head, of 128 outputs, a maximum and a sum
    size = absb.absb_attend_workspace(_layer(), _batch(lens), _rows(new))
    assert size % 256 == 0 and size <= sum(new) * 32 * 65 * 520 + 512
    shared = absb.SharedPrefix([0, len(lens)], [0], AT, AT)       # nothing shared: the same call
    plain = absb.ScoreOpts()
    assert absb.absb_attend_workspace(_layer(), _batch(lens), _rows(new), shared, plain) == absb.absb_attend_workspace(
        _layer(), _batch(lens), _rows(new), None, plain) <= size
    # without options: enough for any window, and for prefixes
    for opts in [absb.ScoreOpts(window=w) for w in (1, 17, 63, 64, 100, 129, 500, 1000, 2047, 4096, 10000, 100000, 2 ** 31 - 1)] + [
            absb.ScoreOpts(window=100, prefix_lens=AT)]:
        assert absb.absb_attend_workspace(_layer(), _batch(lens), _rows(new), None, opts) <= size
    with pytest.raises(absb.AbsbError):
        absb.absb_attend_workspace(_layer(), _batch(lens), _rows(new), None, absb.ScoreOpts(window=-1))


# ------------------------------------------------------------------ requests without rows
def _idle(B, at, new, L, shared=None, opts=absb.ScoreOpts()):
    lens, n = np.zeros(B, np.int32), np.zeros(B, np.int32)
    lens[at], n[at] = L, new
    return absb.absb_attend_workspace(_layer(), _batch(lens), _rows(n), shared, opts)


def test_a_chunk_behind_many_idle_requests_is_planned():
    """65 tiles of 128 rows, 64 of which fill the chip: whichever request of many brings them.  (2080 rows of 32 heads, 524 bytes a
    partial result: no more of them than a cut in 64 of one tile, or in two of all.)"""
    one = _idle(1, 0, 2080, 2080 + (1 << 17))
    assert 0 < one <= 1024 * 128 * 524 + 512
    for B in (40, 64, 1000, 60000, 65535):
        for at in (0, B // 2, B - 1):
            assert _idle(B, at, 2080, 2080 + (1 << 17)) <= 2 * 2080 * 32 * 524 + 512, (B, at)
    assert _idle(63, 62, 2080, 2080 + (1 << 17)) == one


def test_idle_requests_do_not_multiply_the_cuts():
    """One token behind 128 Ki, alone: 64 stretches, 8 x 64 work-groups.  Idle requests' slots are launched as often as the tile is cut."""
    parts = [_idle(B, B - 1, 1, 1 << 17) // (32 * 524) for B in (1, 63, 64, 256, 1000, 60000)]
    assert parts[0] == parts[1] == 64
    assert all(a >= b for a, b in zip(parts, parts[1:])) and parts[2] >= 8 and 999 * 8 * parts[4] < 100000 and 60000 * 8 * parts[5] < 1 << 21


# ------------------------------------------------------------------ limits and what the binding looks at
@pytest.mark.parametrize("n", [(1 << 26) - 3, (1 << 26) - 1])
def test_rotate_store_of_more_rows_than_a_launch_has_threads_for(n):
    """Four rows a work-group of 256 threads: from 2^26 - 3 rows on, 2^32 threads."""
    _refused(absb.ERR_BAD_SHAPE, absb.absb_rotate_store, **_rot(n=n))


def _zeros(*shape, **kw):
    import torch
    kw.setdefault("dtype", torch.float32)
    return torch.zeros(*shape, **kw)


def _torch_types():
    import torch
    return torch.float16, torch.bfloat16, torch.int32, torch.int64, torch.float64


def test_attend_refuses_tensors_shorter_than_the_step():
    """3 rows of 32 heads of two requests: what a call would write or read behind a tensor's end, or beside its rows."""
    f16, bf16, i32, i64, f64 = _torch_types()
    layer, batch, rows = _layer(), _batch((100, 200)), _rows((1, 2))
    short = [dict(lse=_zeros(3, 31)), dict(lse=_zeros(2, 32)), dict(lse=_zeros(3, 64)[:, :32]), dict(lse=_zeros(3, 32, dtype=f16)),
             dict(q=_zeros(3, 32, D)), dict(q=_zeros(3, 32, D, dtype=bf16)), dict(out=_zeros(3, 32, D)), dict(out=_zeros(2, 32, D, dtype=f16)),
             dict(opts=absb.ScoreOpts(slopes=_zeros(31))), dict(opts=absb.ScoreOpts(slopes=_zeros(64)[::2])),
             dict(opts=absb.ScoreOpts(prefix_lens=_zeros(1, dtype=i32))), dict(opts=absb.ScoreOpts(doc_start=_zeros(2, dtype=i32))),
             dict(rows=absb.Rows([0, 1, 3], _zeros(2, dtype=i32))), dict(rows=absb.Rows([0, 3], AT)), dict(rows=absb.Rows([0, 1, 2, 3], AT))]
    for kw in short:
        d = dict(rows=rows, q=AT, out=AT, lse=None, opts=None)
        d.update(kw)
        _refused(absb.ERR_BAD_SHAPE, absb.absb_attend_rows, layer, batch, d["rows"], d["q"], AT, AT, d["out"], d["lse"], d["opts"], BIG_WS)
        _refused(absb.ERR_BAD_SHAPE, absb.absb_attend_shared, layer, batch, d["rows"], absb.SharedPrefix([0, 2], [0], AT, AT), d["q"], AT, AT,
                 d["out"], d["lse"], d["opts"], BIG_WS)
    for r in (absb.Rows([0, 3], AT), absb.Rows([0, 1, 2, 3], AT)):
        with pytest.raises(absb.AbsbError) as e:
            absb.absb_attend_workspace(layer, batch, r)
        assert e.value.status == absb.ERR_BAD_SHAPE
    for shared in (absb.SharedPrefix([0, 2], [0, 0], AT, AT), absb.SharedPrefix([0, 2], [0], _zeros(1, dtype=i32), AT),
                   absb.SharedPrefix([0, 2], [0], AT, _zeros(0, dtype=i32))):
        _refused(absb.ERR_BAD_SHAPE, absb.absb_attend_shared, layer, batch, rows, shared, AT, AT, AT, AT, None, None, BIG_WS)


def test_rotate_and_map_refuse_tensors_shorter_than_the_step():
    f16, bf16, i32, i64, f64 = _torch_types()
    for kw in (dict(freq=_zeros(63, dtype=f64)), dict(freq=_zeros(64)), dict(rope=absb.Rope(rot_dim=66), freq=_zeros(32, dtype=f64)),
               dict(row_pos=_zeros(3, dtype=f16)), dict(row_slot=_zeros(3, dtype=i32)), dict(q=_zeros(3, 32, D)), dict(q=_zeros(3, 32, D, dtype=bf16)),
               dict(q_out=_zeros(3, 32, D)), dict(k=_zeros(3, 8, D)), dict(v=_zeros(3, 8, D, dtype=bf16))):
        _refused(absb.ERR_BAD_SHAPE, absb.absb_rotate_store, **_rot(**kw))
    batch = _batch((5, 6), width=4)
    ring = lambda **kw: absb.PageRing(**dict(dict(pages=_zeros(9, dtype=i32), cursors=_zeros(4, dtype=i64)), **kw))  # noqa: E731
    for kw in (dict(before=_zeros(1, dtype=i32)), dict(off=_zeros(2, dtype=i32)), dict(table=_zeros(1, 4, dtype=i32)), dict(table=_zeros(2, 3, dtype=i32)),
               dict(pos=_zeros(4, dtype=f16)), dict(slot=_zeros(4, dtype=i32)), dict(ring=ring(cursors=_zeros(3, dtype=i64))),
               dict(ring=ring(cursors=_zeros(4, dtype=i32))), dict(ring=ring(pages=_zeros(9, dtype=f16)))):
        d = dict(before=AT, table=AT, off=AT, pos=_T(4), slot=_T(4), ring=None)
        d.update(kw)
        _refused(absb.ERR_BAD_SHAPE, absb.absb_map_rows, _layer(), batch, *d.values())
    _refused(absb.ERR_BAD_SHAPE, absb.absb_map_rows, *_map(batch=batch, ring=ring()), cursors_out=_zeros(3, dtype=i64))


@pytest.mark.parametrize("shared", [absb.SharedPrefix(None, [64], AT, AT), absb.SharedPrefix([0, 2], None, AT, AT)])
def test_attend_shared_without_its_host_arrays(shared):
    _refused(absb.ERR_NULL, absb.absb_attend_shared, _layer(), _batch((100, 200)), _rows((1, 2)), shared, AT, AT, AT, AT, None, None, BIG_WS)


@pytest.mark.parametrize("scale,cap", [(1e9, 1e-30), (3e38, 0.0), (3e38, 1e30)])
def test_attend_refuses_scales_that_binary32_does_not_hold(scale, cap):
    """sm_scale log2(e), and 2 log2(e) sm_scale / cap: infinite, times a score of 0."""
    _refused(absb.ERR_BAD_SHAPE, absb.absb_attend_rows, *_att(layer=_layer(sm_scale=scale), opts=absb.ScoreOpts(softcap=cap), ws=BIG_WS))
