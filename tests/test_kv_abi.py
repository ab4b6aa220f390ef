"""Host-side checks of the cache calls: every refusal comes before any device access."""

import ctypes

import pytest

from paper_2607_13093_amd import _lib

E, U, W = _lib.SPH_E_INVALID_ARG, _lib.SPH_E_UNSUPPORTED, _lib.SPH_E_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def _cache(**kw):
    a = dict(pool=4096, layers=2, layer_stride=1 << 20, n_pages=64, page_stride=17408, table=4096, ld_table=8,
             max_pages=8, lens=4096, refs=4096, n_slots=4, kv_heads=8, head_dim=128, page_tokens=16)
    a.update(kw)
    return _lib.KvCacheStruct(*a.values())


def _ptr(c):
    return None if c is None else ctypes.addressof(c)


@pytest.mark.parametrize("heads,d,page,need", [
    (8, 128, 16, 17408), (1, 64, 16, 1088), (16, 256, 256, 1114112), (0, 128, 16, -1), (8, 96, 16, -1),
    (8, 128, 24, -1), (8, 128, 512, -1), (-1, 64, 16, -1), (70000, 64, 16, -1),
])
def test_page_bytes(lib, heads, d, page, need):
    assert lib.sph_kv_page_bytes(heads, d, page) == need


def _calls(lib, c, layer=0, k=16, v=16, k_row=1024, k_head=128, n=3, R=5, rows=None, slots=None):
    for fn in (lib.sph_kv_append, lib.sph_kv_read):
        yield fn(_ptr(c), layer, k, k_row, k_head, v, k_row, k_head, n, R, rows, slots, None)
    yield lib.sph_kv_attend(_ptr(c), layer, k, k_row, k_head, 8, n, R, rows, slots, 0.1, 0, 0, v, k_row, k_head,
                            None, 4096, 1 << 30, None)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(kv_heads=0), E, b"kv_heads=0"), (dict(head_dim=96), U, b"head_dim=96"),
    (dict(page_tokens=48), U, b"page_tokens=48"), (dict(n_pages=0), E, b"n_pages=0"),
    (dict(layers=0), E, b"layers=0"), (dict(ld_table=7), E, b"ld_table=7"), (dict(n_slots=0), E, b"n_slots=0"),
    (dict(page_stride=17392), E, b"page_stride=17392"), (dict(page_stride=17416), E, b"page_stride=17416"),
    (dict(layer_stride=8), E, b"layer_stride=8"), (dict(pool=None), E, b"NULL"), (dict(table=None), E, b"NULL"),
    (dict(lens=None), E, b"NULL"), (dict(pool=4104), E, b"aligned"),
])
def test_cache_checks(lib, kw, code, msg):
    c = _cache(**kw)
    for rc in _calls(lib, c):
        assert rc == code and msg in lib.sph_last_error(), lib.sph_last_error()
    big = 1 << 30
    for rc in (lib.sph_pages_grow(_ptr(c), 16, 16, 4096, big, None), lib.sph_pages_trim(_ptr(c), 16, None),
               lib.sph_pages_fork(_ptr(c), 16, 16, 1, None), lib.sph_pages_copy(_ptr(c), 16, 16, 1, None),
               lib.sph_pages_compact(_ptr(c), 16, 8, 16, 16, 4096, big, None)):
        assert rc == code and msg in lib.sph_last_error(), lib.sph_last_error()


@pytest.mark.parametrize("kw,msg", [
    (dict(layer=2), b"layer=2"), (dict(layer=-1), b"layer=-1"), (dict(n=-1), b"n_sessions=-1"),
    (dict(n=5), b"beyond n_slots=4"), (dict(n=65536, slots=16), b"n_sessions=65536"), (dict(R=-1), b"R=-1"),
    (dict(R=(1 << 30) + 1), b"R=1073741825"), (dict(k_row=127), b"strides"), (dict(k_head=64), b"strides"),
    (dict(k=None), b"NULL"), (dict(v=None), b"NULL"),
])
def test_row_checks(lib, kw, msg):
    for rc in _calls(lib, _cache(), **kw):
        assert rc == E and msg in lib.sph_last_error(), lib.sph_last_error()


def test_empty_calls_launch_nothing(lib):
    for kw in (dict(n=0), dict(R=0)):
        assert list(_calls(lib, _cache(), k=None, v=None, **kw)) == [0, 0, 0]
    c = _cache()
    assert lib.sph_pages_fork(_ptr(c), None, None, 0, None) == 0
    assert lib.sph_pages_copy(_ptr(c), None, None, 0, None) == 0


@pytest.mark.parametrize("q_heads,scale,window,max_len,ws,nbytes,code,msg", [
    (12, 0.1, 0, 0, 4096, 1 << 30, E, b"q_heads=12"), (0, 0.1, 0, 0, 4096, 1 << 30, E, b"q_heads=0"),
    (8, 0.0, 0, 0, 4096, 1 << 30, E, b"scale"), (8, -1.0, 0, 0, 4096, 1 << 30, E, b"scale"),
    (8, float("nan"), 0, 0, 4096, 1 << 30, E, b"scale"), (8, float("inf"), 0, 0, 4096, 1 << 30, E, b"scale"),
    (8, 0.1, -1, 0, 4096, 1 << 30, E, b"window=-1"), (8, 0.1, 0, -1, 4096, 1 << 30, E, b"max_len=-1"),
])
def test_attend_checks(lib, q_heads, scale, window, max_len, ws, nbytes, code, msg):
    c = _cache(max_pages=4096, ld_table=4096)
    rc = lib.sph_kv_attend(_ptr(c), 0, 16, 2048, 128, q_heads, 1, 5, None, None, scale, window, max_len, 16, 2048, 128,
                           None, ws, nbytes, None)
    assert rc == code and msg in lib.sph_last_error(), lib.sph_last_error()


def test_workspaces(lib):
    c = _cache(max_pages=4096, ld_table=4096)
    p = _ptr(c)
    # one short session needs none, a long one shares its tokens out
    assert lib.sph_kv_attend_workspace(p, 32, 1, 1, 0, 100) == 0
    need = lib.sph_kv_attend_workspace(p, 32, 1, 5, 0, 65536)
    assert need > 0 and lib.sph_kv_attend_workspace(p, 32, 1, 5, 0, 0) == need
    for ws, n in ((None, need), (4096, need - 1), (4104, need)):
        assert lib.sph_kv_attend(p, 0, 16, 4096, 128, 32, 1, 5, None, None, 0.1, 0, 0, 16, 4096, 128, None, ws, n,
                                 None) == W
        assert b"workspace" in lib.sph_last_error()
    for q_heads, n, R, win, most in ((0, 1, 1, 0, 0), (12, 1, 1, 0, 0), (32, 0, 1, 0, 0), (32, 1, 0, 0, 0),
                                     (32, 1, 1, -1, 0), (32, 1, 1, 0, -1)):
        assert lib.sph_kv_attend_workspace(p, q_heads, n, R, win, most) == 0
    assert lib.sph_kv_attend_workspace(None, 32, 1, 1, 0, 0) == 0
    grow, compact = lib.sph_pages_grow_workspace(p), lib.sph_pages_compact_workspace(p)
    assert grow > 0 and compact > 0
    assert lib.sph_pages_grow_workspace(None) == 0 and lib.sph_pages_compact_workspace(None) == 0
    assert lib.sph_pages_grow(p, 16, 16, 4096, grow - 1, None) == W
    assert lib.sph_pages_grow(p, 16, 16, None, grow, None) == W
    assert lib.sph_pages_compact(p, 16, 4096, 16, 16, 4096, compact - 1, None) == W


def test_page_call_checks(lib):
    p, big = _ptr(_cache()), 1 << 30
    keep = _cache()
    p = _ptr(keep)
    for rc, msg in (
            (lib.sph_pages_grow(p, None, 16, 4096, big, None), b"add"),
            (lib.sph_pages_grow(p, 16, None, 4096, big, None), b"status_out"),
            (lib.sph_pages_trim(p, None, None), b"kept"),
            (lib.sph_pages_fork(p, None, 16, 1, None), b"parents"),
            (lib.sph_pages_fork(p, 16, 16, 5, None), b"n=5"),
            (lib.sph_pages_fork(p, 16, 16, -1, None), b"n=-1"),
            (lib.sph_pages_copy(p, 16, None, 1, None), b"dst"),
            (lib.sph_pages_copy(p, 16, 16, 65, None), b"n=65"),
            (lib.sph_pages_compact(p, None, 8, 16, 16, 4096, big, None), b"output"),
            (lib.sph_pages_compact(p, 16, 7, 16, 16, 4096, big, None), b"ld_out=7")):
        assert rc == E, msg
    assert b"ld_out=7" in lib.sph_last_error()
    no_refs = _cache(refs=None)
    assert lib.sph_pages_trim(_ptr(no_refs), 16, None) == E and b"refs" in lib.sph_last_error()
