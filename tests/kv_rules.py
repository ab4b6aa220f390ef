"""How a cache attention call is shared out, asked of the built library's own rule
(a host function, no GPU)."""

import ctypes

from paper_2607_13093_amd import _lib


def attend_shape(d, sessions, R, kv_heads, q_heads, max_len, window=0):
    """(row tiles of a wave, waves that share its rows, workgroups for the rows of a
    head, shares of the tokens, tokens of a share)."""
    f = _lib.load()["_ZN3sph15kv_attend_shapeEillllllPi"]
    f.argtypes, f.restype = [ctypes.c_int] + [ctypes.c_int64] * 6 + [ctypes.c_void_p], None
    out = (ctypes.c_int * 5)()
    f(d, sessions, R, kv_heads, q_heads, max_len, window, out)
    return tuple(out)


def join_kind(splits):
    """0: no join, 1: a row's shares by one group of lanes, 2: by a workgroup."""
    return 0 if splits == 1 else 1 if splits <= 8 else 2
