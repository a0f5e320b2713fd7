"""Calls that zoact_linear_rows and the cache's entry points refuse on the host, before anything reaches the
GPU (these make no HIP call, so they run without one)."""
import ctypes

import pytest

from paper_2607_01125_amd import zoact as Z

P = ctypes.c_void_p(256)
ODD = ctypes.c_void_p(258)


def _lin(**kw):
    f = dict(w_dtype=Z.INT4_G128, w=256, w_scales=256, bias=None, ut=None, d_in=256, d_out=64, r=0, coef_offset=0)
    f.update(kw)
    return Z.LinearDesc(**f)


def _rows(lin, rows=4, x=P, p=None, res=None, flags=0, y=P, yd=Z.BF16, arena=None):
    return Z.lib().zoact_linear_rows(ctypes.byref(lin), ctypes.byref(arena) if arena else None, x, rows, p, res, flags,
                                     y, yd, None)


ARENA = Z.ArenaDesc(Z.BF16, 256, 256, 256, 64 * 8)


@pytest.mark.parametrize("call,word", [
    (lambda: _rows(_lin(), rows=0), b"rows=0"),
    (lambda: _rows(_lin(), rows=65), b"rows=65"),
    (lambda: _rows(_lin(), x=None), b"NULL"),
    (lambda: _rows(_lin(w=None)), b"NULL"),
    (lambda: _rows(_lin(w_scales=None)), b"w_scales"),
    (lambda: _rows(_lin(d_in=192)), b"d_in"),
    (lambda: _rows(_lin(d_in=0)), b"d_in"),
    (lambda: _rows(_lin(d_out=40)), b"d_out"),
    (lambda: _rows(_lin(d_out=48), flags=Z.EPI_SWIGLU), b"d_out"),
    (lambda: _rows(_lin(), flags=Z.SHARED_X), b"flags"),
    (lambda: _rows(_lin(), flags=Z.EPI_SWIGLU | Z.EPI_RELU), b"exclusive"),
    (lambda: _rows(_lin(), yd=7), b"y must be"),
    (lambda: _rows(_lin(), x=ODD), b"aligned"),
    (lambda: _rows(_lin(), res=ODD), b"aligned"),
    (lambda: _rows(_lin(ws=258)), b"aligned"),
    (lambda: _rows(_lin(r=8), arena=ARENA), b"needs p"),
    (lambda: _rows(_lin(r=8), p=P), b"arena"),
    (lambda: _rows(_lin(r=257), p=P, arena=ARENA), b"r=257"),
    (lambda: _rows(_lin(r=8, coef_offset=1), p=P, arena=ARENA), b"outside the arena"),
    (lambda: _rows(_lin(r=8, coef_offset=-1), p=P, arena=ARENA), b"outside the arena"),
    (lambda: _rows(_lin(r=8, plain_begin=10, plain_end=65), p=P, arena=ARENA), b"plain range"),
    (lambda: _rows(_lin(r=8, plain_begin=10, plain_end=9), p=P, arena=ARENA), b"plain range"),
])
def test_linear_rows_refuses(call, word):
    assert call() == Z.E_INVALID
    assert word in Z.lib().zoact_last_error(), Z.lib().zoact_last_error()


def test_linear_rows_takes_int4_only():
    assert _rows(_lin(w_dtype=Z.BF16)) == Z.E_UNSUPPORTED


def _cache(**kw):
    f = dict(k=256, v=256, k_scale=256, v_scale=256, table=256, len=256, refs=256, n_pages=10, n_layers=2, n_kv_heads=2,
             head_dim=64, n_slots=4, max_pages=3)
    f.update(kw)
    return Z.CacheDesc(**f)


def _batch(**kw):
    f = dict(n=2, max_new=1, rows=2, slots=None, row_begin=None, pos=256, status=None)
    f.update(kw)
    return Z.CacheBatchDesc(**f)


BIG = 1 << 30


def _extend(c=None, b=None, ws=P, nb=BIG):
    return Z.lib().zoact_cache_extend(ctypes.byref(c or _cache()), ctypes.byref(b or _batch()), ws, nb, None)


def _append(c=None, b=None, layer=0, k=P, ldk=128, v=P, ldv=128, dt=Z.BF16, cos=None, sin=None, n_pos=0):
    return Z.lib().zoact_cache_append(ctypes.byref(c or _cache()), layer, k, ldk, v, ldv, dt, ctypes.byref(b or _batch()),
                                      cos, sin, n_pos, None)


def _attend(c=None, b=None, layer=0, q=P, ldq=256, dt=Z.BF16, H=4, max_len=10, cos=None, sin=None, n_pos=0, out=P, ws=None,
            nb=0):
    return Z.lib().zoact_attention_cache(ctypes.byref(c or _cache()), layer, q, ldq, dt, H, ctypes.byref(b or _batch()),
                                         1.0, max_len, cos, sin, n_pos, out, ws, nb, None)


BAD_CACHES = [_cache(k=None), _cache(refs=None), _cache(k=264), _cache(v_scale=260), _cache(table=258), _cache(n_pages=0),
              _cache(n_pages=2 ** 31), _cache(n_layers=0), _cache(n_layers=40000), _cache(n_kv_heads=0),
              _cache(n_kv_heads=70000), _cache(head_dim=96), _cache(n_slots=0), _cache(max_pages=0),
              _cache(max_pages=2 ** 25)]
BAD_BATCHES = [_batch(n=0), _batch(n=1025), _batch(n=5), _batch(max_new=0), _batch(rows=-1), _batch(rows=2 ** 31),
               _batch(rows=1), _batch(pos=None), _batch(n=4, max_new=3, rows=11)]


@pytest.mark.parametrize("i", range(len(BAD_CACHES)))
def test_every_call_refuses_a_cache_that_is_none(i):
    c, L = BAD_CACHES[i], Z.lib()
    assert _extend(c) == Z.E_INVALID
    assert _append(c) == Z.E_INVALID
    assert _attend(c) == Z.E_INVALID
    assert L.zoact_cache_fork(ctypes.byref(c), P, P, 1, P, BIG, None, None) == Z.E_INVALID
    assert L.zoact_cache_free(ctypes.byref(c), P, 1, None, None) == Z.E_INVALID
    assert L.zoact_cache_compact(ctypes.byref(c), P, BIG, None, None) == Z.E_INVALID


@pytest.mark.parametrize("i", range(len(BAD_BATCHES)))
def test_every_call_refuses_a_batch_that_is_none(i):
    for f in (_extend, _append, _attend):
        assert f(b=BAD_BATCHES[i]) == Z.E_INVALID
        assert b"batch" in Z.lib().zoact_last_error()


@pytest.mark.parametrize("field", ["pos", "slots", "row_begin", "status"])
def test_every_call_refuses_misaligned_batches(field):
    for f in (_extend, _append, _attend):
        assert f(b=_batch(**{field: 258})) == Z.E_INVALID
        assert b"aligned" in Z.lib().zoact_last_error()


def test_a_batch_of_no_rows_is_served_without_buffers():
    b = _batch(rows=0, row_begin=256)
    assert _append(b=b, k=None, v=None) == Z.OK and _attend(b=b, q=None, out=None) == Z.OK
    assert _append(b=b, k=None, v=None, layer=2) == Z.E_INVALID and _attend(b=b, q=None, out=None, H=3) == Z.E_INVALID
    assert _append(k=None) == Z.E_INVALID and _attend(out=None) == Z.E_INVALID


def test_lengths_past_the_table_do_not_enlarge_the_workspace():
    f = lambda n: Z.lib().zoact_attention_cache_workspace_bytes(ctypes.byref(_cache(max_pages=4096)),
                                                                ctypes.byref(_batch()), 4, n)
    assert f(4096 * 64) == f(2 ** 63 - 1) > 0


def test_workspaces():
    need = Z.lib().zoact_cache_workspace_bytes(ctypes.byref(_cache()))
    assert need > 0
    assert _extend(nb=need - 1) == Z.E_WORKSPACE and _extend(ws=None) == Z.E_WORKSPACE
    assert _extend(ws=ODD, nb=need) == Z.E_INVALID
    L, c = Z.lib(), ctypes.byref(_cache())
    assert L.zoact_cache_fork(c, P, P, 1, P, need - 1, None, None) == Z.E_WORKSPACE
    assert L.zoact_cache_compact(c, None, need, None, None) == Z.E_WORKSPACE
    big = _cache(n_pages=10 ** 6)
    assert L.zoact_cache_workspace_bytes(ctypes.byref(big)) >= 12 * 10 ** 6


def test_slots():
    L, c = Z.lib(), ctypes.byref(_cache())
    for n in (0, -1, 5):
        assert L.zoact_cache_fork(c, P, P, n, P, BIG, None, None) == Z.E_INVALID
        assert L.zoact_cache_free(c, P, n, None, None) == Z.E_INVALID
    assert L.zoact_cache_fork(c, None, P, 1, P, BIG, None, None) == Z.E_INVALID
    assert L.zoact_cache_free(c, None, 1, None, None) == Z.E_INVALID


@pytest.mark.parametrize("call", [
    lambda: _append(layer=2), lambda: _append(layer=-1), lambda: _append(k=None), lambda: _append(k=ODD),
    lambda: _append(ldk=120), lambda: _append(ldv=132), lambda: _append(dt=2), lambda: _append(dt=Z.F32, ldk=130),
    lambda: _append(cos=P), lambda: _append(sin=P, n_pos=4), lambda: _append(cos=P, sin=P, n_pos=0),
    lambda: _attend(layer=2), lambda: _attend(q=None), lambda: _attend(out=ODD), lambda: _attend(H=3), lambda: _attend(H=0),
    lambda: _attend(ldq=248), lambda: _attend(ldq=260), lambda: _attend(dt=5), lambda: _attend(max_len=0),
    lambda: _attend(cos=P, n_pos=4), lambda: _attend(cos=P, sin=P, n_pos=-1),
    lambda: _attend(b=_batch(n=1, max_new=2 ** 30, rows=2 ** 30)),
    lambda: _extend(b=_batch(n=1024, max_new=2 ** 30, rows=2 ** 30, row_begin=256, slots=256)),
])
def test_rows_and_tables(call):
    assert call() == Z.E_INVALID


def test_lists_and_words_that_are_misaligned():
    """A status word off its four bytes would fault in the atomic that sets a bit."""
    L, c = Z.lib(), ctypes.byref(_cache())
    for a in range(3):
        src, dst, status = (ODD if a == i else P for i in range(3))
        assert L.zoact_cache_fork(c, src, dst, 1, P, BIG, status, None) == Z.E_INVALID
        assert b"aligned" in L.zoact_last_error()
    for slots, status in ((ODD, P), (P, ODD)):
        assert L.zoact_cache_free(c, slots, 1, status, None) == Z.E_INVALID
        assert b"aligned" in L.zoact_last_error()
    assert L.zoact_cache_compact(c, P, BIG, ODD, None) == Z.E_INVALID
    assert b"aligned" in L.zoact_last_error()


def test_more_features_than_a_launch_has_threads_for():
    for rows in (1, 20, 64):
        assert _rows(_lin(d_in=128, d_out=1 << 29), rows=rows) == Z.E_INVALID
        assert b"d_out" in Z.lib().zoact_last_error()
