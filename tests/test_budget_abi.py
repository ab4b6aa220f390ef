"""Host-side checks of eviction, token weights and shared attention: every refusal comes
before any device access."""

import ctypes

import pytest

from paper_2607_13093_amd import _lib

E, U, W = _lib.SPH_E_INVALID_ARG, _lib.SPH_E_UNSUPPORTED, _lib.SPH_E_WORKSPACE
BIG = 1 << 30


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


BAD_CACHES = [
    (dict(kv_heads=0), E, b"kv_heads=0"), (dict(head_dim=96), U, b"head_dim=96"),
    (dict(page_tokens=48), U, b"page_tokens=48"), (dict(n_pages=0), E, b"n_pages=0"),
    (dict(layers=0), E, b"layers=0"), (dict(ld_table=7), E, b"ld_table=7"), (dict(n_slots=0), E, b"n_slots=0"),
    (dict(page_stride=17392), E, b"page_stride=17392"), (dict(layer_stride=8), E, b"layer_stride=8"),
    (dict(pool=None), E, b"NULL"), (dict(table=None), E, b"NULL"), (dict(lens=None), E, b"NULL"),
    (dict(pool=4104), E, b"aligned"),
]


def _evict(lib, c, w=16, ld=128, keep=16, first=0, recent=0, out=16, ld_out=128, kept=16, ld_kept=128, ws=4096, n=BIG):
    return lib.sph_pages_evict(_ptr(c), w, ld, keep, first, recent, out, ld_out, kept, ld_kept, ws, n, None)


@pytest.mark.parametrize("kw,code,msg", BAD_CACHES + [(dict(refs=None), E, b"NULL")])
def test_evict_cache_checks(lib, kw, code, msg):
    c = _cache(**kw)
    assert _evict(lib, c) == code and msg in lib.sph_last_error(), lib.sph_last_error()
    assert _evict(lib, None) == E


@pytest.mark.parametrize("kw,code,msg", [
    (dict(w=None), E, b"NULL"), (dict(keep=None), E, b"NULL"), (dict(out=None), E, b"NULL"),
    (dict(first=-1), E, b"first=-1"), (dict(recent=-1), E, b"recent=-1"), (dict(ld=127), E, b"ld_weights=127"),
    (dict(ld_out=127), E, b"ld_out=127"), (dict(ld_kept=127), E, b"ld_kept=127"),
    (dict(ld_out=130), E, b"in place"), (dict(ws=None), W, b"workspace"), (dict(ws=4104), W, b"workspace"),
    (dict(n=8), W, b"workspace"),
])
def test_evict_checks(lib, kw, code, msg):
    c = _cache()
    assert _evict(lib, c, **kw) == code and msg in lib.sph_last_error(), lib.sph_last_error()


def test_evict_workspace(lib):
    c = _cache()
    need = lib.sph_pages_evict_workspace(_ptr(c))
    assert need >= 4 * 128 * 8
    assert lib.sph_pages_evict_workspace(None) == 0 and lib.sph_pages_evict_workspace(_ptr(_cache(head_dim=96))) == 0
    assert _evict(lib, c, n=need - 1) == W
    # sizes past what there is are refused, not wrapped
    huge = _cache(n_slots=(1 << 31) - 1, max_pages=1 << 27, ld_table=1 << 27)
    assert _evict(lib, huge, ld=1 << 30, ld_out=1 << 30, kept=None, n=(1 << 63)) == W
