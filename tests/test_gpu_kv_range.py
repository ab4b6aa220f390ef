"""Ends of the cache attention's argument range on the GPU, against the oracle within
the bounds derived in test_gpu_kv.py."""

import numpy as np
import pytest

import paper_2607_13093_amd as sph

from kv_build import bf16, filled, host
from test_gpu_kv import _check, say

pytestmark = pytest.mark.gpu

WIDE = [(1 << 30) - 1, 1 << 30, (1 << 31) - 1, 1 << 31, 1 << 40]


@pytest.mark.parametrize("window", WIDE)
@pytest.mark.parametrize("hq,d,R,lens,hint", [
    (1, 64, 9, [3, 0, 40], 0),                     # more rows than tokens
    (8, 128, 9, [3, 700], 65536),                  # the same, and the tokens shared out
    (8, 256, 130, [2, 129], 0),
    (4, 128, 5, [5000], 5000),
])
def test_windows_beyond_every_length_are_none(hq, d, R, lens, hint, window):
    say("wide window", hq, d, R, lens, hint, window)
    rng = np.random.default_rng(R + d)
    c, k, v = filled(rng, lens, 1, d, 16, extra=4096 if hint > 5000 else 1)
    q, q64 = bf16(rng, len(lens) * R, hq, d, scale=2.0)
    _check(c, q, q64, k, v, R, d ** -0.5, lens, window=window, max_len=hint)
    out, lse = sph.kv_attend(c, 0, q, R, d ** -0.5, window=window, max_len=hint, want_lse=True)
    none, lse0 = sph.kv_attend(c, 0, q, R, d ** -0.5, max_len=hint, want_lse=True)
    np.testing.assert_array_equal(host(out), host(none))
    np.testing.assert_array_equal(host(lse), host(lse0))
