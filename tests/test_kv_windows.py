"""Wide windows of the cache attention, as far as the host decides about them (no GPU)."""

import ctypes

import pytest

from paper_2607_13093_amd import _lib


def _cache(d, kv_heads, capacity):
    """A cache whose slots hold `capacity` tokens, in pages of 16."""
    return _lib.KvCacheStruct(pool=4096, layers=1, layer_stride=0, n_pages=64, page_stride=17 * d * kv_heads, table=4096,
                              ld_table=capacity // 16, max_pages=capacity // 16, lens=4096, refs=4096, n_slots=64,
                              kv_heads=kv_heads, head_dim=d, page_tokens=16)


SIZES = [  # d, kv heads, q heads, sessions, rows, max_len: all share their tokens out
    (64, 4, 20, 33, 33, 11348), (128, 4, 16, 33, 33, 123547), (64, 2, 16, 16, 100, 16001), (128, 8, 32, 1, 5, 65521),
    (256, 2, 6, 2, 9, 30000),
]


@pytest.mark.parametrize("window", [1 << 31, 1 << 40])
@pytest.mark.parametrize("d,hkv,hq,n,R,most", SIZES)
def test_a_call_takes_the_workspace_that_its_query_asks_for(d, hkv, hq, n, R, most, window):
    # a window beyond every length is none, in the query as in the call
    lib = _lib.load()
    c = _cache(d, hkv, 1 << 17)
    p = ctypes.addressof(c)
    need = lib.sph_kv_attend_workspace(p, hq, n, R, 0, most)
    assert need > 0
    assert lib.sph_kv_attend_workspace(p, hq, n, R, window, most) == need
    # refused before anything is launched; the message says what the call needs
    rc = lib.sph_kv_attend(p, 0, 16, hq * d, d, hq, n, R, None, None, 0.1, window, most, 16, hq * d, d, None, 4096,
                           need - 1, None)
    assert rc == _lib.SPH_E_WORKSPACE and f"need {need} ".encode() in lib.sph_last_error()
