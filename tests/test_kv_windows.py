"""Wide windows of the cache attention, as far as the host decides about them (no GPU)."""

import ctypes
import random

import pytest

import kv_rules
from paper_2607_13093_amd import _lib

MOST = 1 << 30                                     # tokens of a session


def _window(window, most):
    """What a call makes of its window where no session holds more than `most` tokens."""
    f = _lib.load()["_ZN3sph9kv_windowEll"]
    f.argtypes, f.restype = [ctypes.c_int64] * 2, ctypes.c_int64
    return f(window, most)


def _span(base, r_lo, r_hi, window, split=0, splits=1, chunk=32):
    """lo, hi, all_lo, all_hi, from, to: as the kernel works them out, in 32 bits."""
    f = _lib.load()["_ZN3sph14kv_attend_spanEiiiiiiiPi"]
    f.argtypes, f.restype = [ctypes.c_int] * 7 + [ctypes.c_void_p], None
    out = (ctypes.c_int * 6)()
    f(base, r_lo, r_hi, window, split, splits, chunk, out)
    return tuple(out)


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


WIDE = [MOST - 1, MOST, MOST + 1, (1 << 31) - 1, 1 << 31, 1 << 40]


@pytest.mark.parametrize("window", WIDE)
def test_a_window_as_long_as_a_slot_is_none(window):
    for most in (16, 1 << 17, MOST):
        assert _window(window, most) == (window if window < most else 0)
    assert _window(0, 16) == 0 and _window(15, 16) == 15 and _window(16, 16) == 0
    lib = _lib.load()
    for d, hkv, hq, n, R, most in SIZES:           # the sharing out is that of no window, too
        p = ctypes.addressof(c := _cache(d, hkv, 1 << 17))
        assert lib.sph_kv_attend_workspace(p, hq, n, R, window, most) == lib.sph_kv_attend_workspace(p, hq, n, R, 0, most)


@pytest.mark.parametrize("window", [0, 1, 31, 1000] + WIDE)
@pytest.mark.parametrize("n,rows", [(3, 9), (0, 5), (1, 1), (7, 7), (5000, 3), (40, 4099), (MOST, 1), (MOST, MOST), (0, MOST),
                                    (MOST - 5, 100)])
def test_tokens_seen(n, rows, window):
    # against whole numbers of any size
    w = _window(window, MOST)
    base = n - rows
    for r_lo, r_hi in ((0, 0), (0, min(rows - 1, 63)), (rows - 1, rows - 1), (rows // 2, min(rows // 2 + 15, rows - 1))):
        lo, hi, all_lo, all_hi, first, end = _span(base, r_lo, r_hi, w)
        assert hi == max(0, base + r_hi + 1) and all_hi == max(0, base + r_lo + 1)
        start = base + r_lo - window + 1 if window else 0
        assert lo == max(0, start) // 32 * 32
        # whole tiles begin where the last row does; below 0 it does not matter where
        assert max(all_lo, 0) == max(0, base + r_hi - window + 1 if window else 0)
        assert (first, end) == (lo, hi)


def test_shares_cover_what_is_seen():
    rng = random.Random(9)
    for _ in range(5000):
        d, hkv, g = rng.choice([64, 128, 256]), rng.choice([1, 2, 8]), rng.choice([1, 3, 8])
        sessions, R = rng.choice([1, 2, 16, 64]), rng.choice([1, 2, 9, 100, 4099])
        most = rng.choice([16, 700, 16001, 123547, MOST - 7, MOST])
        n = rng.choice([0, 1, 3, rng.randint(0, most), most])
        window = _window(rng.choice([0, 1, 50, 1024] + WIDE), MOST)
        hint = rng.choice([most, 1, MOST])         # a wrong hint may not lose tokens
        mt, wt, tiles, splits, chunk = kv_rules.attend_shape(d, sessions, R, hkv, hkv * g, hint, window)
        per = 16 * mt * ((8 if wt == 8 else 4) // wt)
        for tile in {0, tiles // 2, tiles - 1}:
            r_lo, r_hi = tile * per // g, (min(tile * per + per, R * g) - 1) // g
            shares = [_span(n - R, r_lo, r_hi, window, k, splits, chunk) for k in range(splits)]
            lo, hi = shares[0][:2]
            at = lo
            for share in shares:
                first, end = share[4:]
                assert 0 <= first <= (1 << 31) - 1 - 256 * 32
                if first >= hi:
                    assert end <= first
                    continue
                assert first == at and first < end <= hi
                at = end
            assert at == max(hi, lo)
