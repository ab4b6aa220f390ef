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


def _weigh(lib, c, layer=0, q=16, q_row=4096, q_head=128, q_heads=32, lse=16, n=3, R=5, rows=None, slots=None, scale=0.1,
           window=0, max_len=0, fresh=0, w=16, ld=128, ws=4096, nb=BIG):
    return lib.sph_kv_weigh(_ptr(c), layer, q, q_row, q_head, q_heads, lse, n, R, rows, slots, scale, window, max_len,
                            fresh, w, ld, ws, nb, None)


@pytest.mark.parametrize("kw,code,msg", BAD_CACHES)
def test_weigh_cache_checks(lib, kw, code, msg):
    c = _cache(**kw)
    assert _weigh(lib, c) == code and msg in lib.sph_last_error(), lib.sph_last_error()
    assert _weigh(lib, None) == E


@pytest.mark.parametrize("kw,code,msg", [
    (dict(layer=2), E, b"layer=2"), (dict(layer=-1), E, b"layer=-1"), (dict(n=-1), E, b"n_sessions=-1"),
    (dict(n=5), E, b"beyond n_slots=4"), (dict(R=-1), E, b"R=-1"), (dict(q_heads=12), E, b"q_heads=12"),
    (dict(q_heads=0), E, b"q_heads=0"), (dict(scale=0.0), E, b"scale"), (dict(scale=float("nan")), E, b"scale"),
    (dict(scale=2e6), E, b"scale"), (dict(window=-1), E, b"window=-1"), (dict(max_len=-1), E, b"max_len=-1"),
    (dict(q_row=127), E, b"strides"), (dict(q_head=64), E, b"strides"), (dict(ld=127), E, b"ld_weights=127"),
    (dict(R=1 << 30, n=1), U, b"rows of 4 heads"), (dict(q=None), E, b"NULL"), (dict(lse=None), E, b"NULL"),
    (dict(w=None), E, b"NULL"), (dict(ws=None), W, b"workspace"), (dict(ws=4104), W, b"workspace"),
    (dict(nb=8), W, b"workspace"),
])
def test_weigh_checks(lib, kw, code, msg):
    c = _cache()
    assert _weigh(lib, c, **kw) == code and msg in lib.sph_last_error(), lib.sph_last_error()


def test_weigh_workspace_and_empty_calls(lib):
    c = _cache()
    p = _ptr(c)
    need = lib.sph_kv_weigh_workspace(p, 32, 3, 5, 0)
    assert need > 0 and _weigh(lib, c, nb=need - 1) == W
    for bad in ((None, 32, 3, 5, 0), (p, 12, 3, 5, 0), (p, 32, 0, 5, 0), (p, 32, 3, 0, 0), (p, 32, 3, 5, -1)):
        assert lib.sph_kv_weigh_workspace(*bad) == 0
    # many sessions fill the device by their tokens alone
    assert lib.sph_kv_weigh_workspace(_ptr(_cache(n_slots=4096)), 32, 4096, 1, 0) == 0
    for kw in (dict(n=0), dict(R=0)):
        assert _weigh(lib, c, q=None, lse=None, w=None, ws=None, nb=0, **kw) == 0


def _share(lib, c, q_heads=32, n=3, R=5, rows=None, slots=None, window=0, max_len=0, plan=4096, nb=BIG):
    return lib.sph_kv_share(_ptr(c), q_heads, n, R, rows, slots, window, max_len, plan, nb, None)


def _shared(lib, c, layer=0, q=16, q_row=4096, q_head=128, q_heads=32, n=3, R=5, rows=None, slots=None, scale=0.1, window=0,
            max_len=0, plan=4096, plan_bytes=BIG, out=16, o_row=4096, o_head=128, lse=None, ws=4096, nb=BIG):
    return lib.sph_kv_attend_shared(_ptr(c), layer, q, q_row, q_head, q_heads, n, R, rows, slots, scale, window, max_len, plan,
                                    plan_bytes, out, o_row, o_head, lse, ws, nb, None)


@pytest.mark.parametrize("kw,code,msg", BAD_CACHES)
def test_share_cache_checks(lib, kw, code, msg):
    c = _cache(**kw)
    for call in (_share, _shared):
        assert call(lib, c) == code and msg in lib.sph_last_error(), lib.sph_last_error()
        assert call(lib, None) == E


BOTH = [
    (dict(n=-1), E, b"n_sessions=-1"), (dict(n=5), E, b"beyond n_slots=4"), (dict(R=-1), E, b"R=-1"),
    (dict(q_heads=12), E, b"q_heads=12"), (dict(q_heads=0), E, b"q_heads=0"), (dict(window=-1), E, b"window=-1"),
    (dict(max_len=-1), E, b"max_len=-1"), (dict(n=2049, slots=16), U, b"2048 sessions"), (dict(R=1 << 24), U, b"2^26 rows"),
]


@pytest.mark.parametrize("kw,code,msg", BOTH + [
    (dict(plan=None), W, b"workspace"), (dict(plan=4104), W, b"workspace"), (dict(nb=100), W, b"workspace")])
def test_share_checks(lib, kw, code, msg):
    c = _cache()
    assert _share(lib, c, **kw) == code and msg in lib.sph_last_error(), lib.sph_last_error()


@pytest.mark.parametrize("kw,code,msg", BOTH + [
    (dict(layer=2), E, b"layer=2"), (dict(scale=0.0), E, b"scale"), (dict(scale=float("inf")), E, b"scale"),
    (dict(q_row=127), E, b"strides"), (dict(q_head=64), E, b"strides"), (dict(o_row=127), E, b"strides"),
    (dict(q=None), E, b"NULL"), (dict(out=None), E, b"NULL"), (dict(plan=None), E, b"plan"), (dict(plan=4104), E, b"plan"),
    (dict(plan_bytes=100), E, b"plan"), (dict(ws=None), W, b"workspace"), (dict(ws=4104), W, b"workspace"),
    (dict(nb=100), W, b"workspace")])
def test_shared_attention_checks(lib, kw, code, msg):
    c = _cache()
    assert _shared(lib, c, **kw) == code and msg in lib.sph_last_error(), lib.sph_last_error()


def test_share_sizes_and_empty_calls(lib):
    c = _cache()
    p = _ptr(c)
    plan, ws = lib.sph_kv_share_bytes(p, 32, 3, 5, 0), lib.sph_kv_attend_shared_workspace(p, 32, 3, 5, 0)
    assert plan > 0 and ws >= 3 * 5 * 32 * 2 * (128 * 4 + 8)
    assert _share(lib, c, nb=plan - 1) == W and _shared(lib, c, plan_bytes=plan - 1) == E and _shared(lib, c, nb=ws - 1) == W
    for bad in ((None, 32, 3, 5, 0), (p, 12, 3, 5, 0), (p, 32, 0, 5, 0), (p, 32, 3, 0, 0), (p, 32, 3, 5, -1),
                (p, 32, 2049, 5, 0), (p, 32, 3, 1 << 24, 0)):
        assert lib.sph_kv_share_bytes(*bad) == 0 and lib.sph_kv_attend_shared_workspace(*bad) == 0
    for kw in (dict(n=0), dict(R=0)):
        assert _share(lib, c, plan=None, nb=0, **kw) == 0
        assert _shared(lib, c, q=None, out=None, plan=None, plan_bytes=0, ws=None, nb=0, **kw) == 0
