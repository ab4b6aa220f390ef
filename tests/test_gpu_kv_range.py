"""Ends of the cache attention's argument range on the GPU, against the oracle within
the bounds derived in test_gpu_kv.py."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph
from oracle import kv_cache as O

from kv_build import bf16, cache_of, filled, host
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


# ---- scores of any size ------------------------------------------------------

@pytest.mark.parametrize("hq,hkv,d,R,lens,window", [
    (4, 1, 64, 5, [5, 200], 0), (8, 2, 128, 3, [7, 90, 300], 0), (8, 1, 128, 5, [9000], 0),   # the last in shares
    (4, 1, 256, 9, [40, 513], 0), (2, 1, 128, 70, [70, 400], 33),
])
def test_rows_of_scores_far_below_zero(hq, hkv, d, R, lens, window):
    # every product is negative, sums of some -1e35: a softmax like any other at a scale that fits
    say("far below zero", hq, hkv, d, R, lens, window)
    rng = np.random.default_rng(d + R)
    c = cache_of(rng, lens, hkv, d, 16)
    n, L = len(lens), max(lens)
    k, k64 = bf16(rng, n * L, hkv, d)
    v, v64 = bf16(rng, n * L, hkv, d)
    k, k64 = k.abs() * 2.0 ** 50, np.abs(k64) * 2.0 ** 50
    sph.kv_append(c, 0, k, v, L, rows=torch.tensor(lens, dtype=torch.int32).cuda())
    keys, values = ([O.quantize(x.reshape(n, L, hkv, d)[s, :lens[s]]) for s in range(n)] for x in (k64, v64))
    q, q64 = bf16(rng, n * R, hq, d)
    q, q64 = -q.abs() * 2.0 ** 60, -np.abs(q64) * 2.0 ** 60
    _check(c, q, q64, keys, values, R, 2.0 ** -108, lens, window=window)


def _one_dimension(rng, q0, k0, d=128, hint=0):
    """Queries [R] and keys [n] along the first dimension alone: (cache, q, values as held)."""
    c = cache_of(rng, [len(k0)], 1, d, 16, extra=hint // 16 + 1)
    k = torch.zeros(len(k0), 1, d, dtype=torch.bfloat16)
    k[:, 0, 0] = torch.tensor(k0).to(torch.bfloat16)
    v, v64 = bf16(rng, len(k0), 1, d)
    sph.kv_append(c, 0, k.cuda(), v, len(k0))
    q = torch.zeros(len(q0), 1, d, dtype=torch.bfloat16)
    q[:, 0, 0] = torch.tensor(q0).to(torch.bfloat16)
    return c, q.cuda(), O.quantize(v64)


@pytest.mark.parametrize("hint", [0, 1 << 16])       # in one share of the tokens, in many
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -40, 2.0 ** 19])
def test_the_largest_score_takes_all_however_low(scale, hint):
    # scores are exact (or below fp32), the nearest two differ by more than it can weigh
    say("one takes all", scale, hint)
    rng = np.random.default_rng(77)
    k0 = [float(2.0 ** x) for x in (20, 14, 19, 16, 11, 30, 12, 40)] + [2.0 ** 33] * 100
    q0 = [-(2.0 ** 60), -(2.0 ** 90) if scale <= 1 else -(2.0 ** 70)]
    c, q, values = _one_dimension(rng, q0, k0, hint=hint)
    out, lse = sph.kv_attend(c, 0, q, 2, scale, max_len=hint, want_lse=True)
    for r, x in enumerate(q0):
        np.testing.assert_array_equal(host(out)[r, 0], values[4, 0])
        want = scale * x * 2.0 ** 11
        assert abs(host(lse)[r, 0] - want) <= 2.0 ** -20 * abs(want)


@pytest.mark.parametrize("hint", [0, 1 << 16])
def test_scores_beyond_fp32(hint):
    # above: the row answers NaN; below: no weight, a row of nothing else is one that sees nothing
    say("beyond fp32", hint)
    rng = np.random.default_rng(78)
    k0 = [2.0 ** 20, 2.0 ** 26, 0.0] + [2.0 ** 26] * 70
    c, q, values = _one_dimension(rng, [2.0 ** 100, -(2.0 ** 100), 2.0 ** -30], k0, hint=hint)
    out, lse = (host(x) for x in sph.kv_attend(c, 0, q, 3, 2.0 ** 19, max_len=hint, want_lse=True))
    assert np.isnan(out[0]).all() and np.isnan(lse[0]).all()
    # the token with a key of zero takes all
    np.testing.assert_array_equal(out[1, 0], values[2, 0])
    assert lse[1, 0] == 0
    assert np.isfinite(out[2]).all() and np.isfinite(lse[2]).all()
    c, q, _ = _one_dimension(rng, [-(2.0 ** 100)], [2.0 ** 26] * 40, hint=hint)
    out, lse = (host(x) for x in sph.kv_attend(c, 0, q, 1, 2.0 ** 19, max_len=hint, want_lse=True))
    assert not out.any() and np.isneginf(lse).all()


# ---- lengths of any size -----------------------------------------------------

@pytest.mark.parametrize("d,page,R,window", [(64, 16, 3, 0), (128, 64, 1, 0), (128, 16, 70, 0), (256, 32, 5, 40)])
@pytest.mark.parametrize("length", [(1 << 31) - 1, 1 << 30, 0])
def test_lengths_beyond_a_slot_s_row_are_cut_to_it(d, page, R, window, length):
    # every page of the row is written, so that a wrong cut shows
    say("length", length, d, page, R, window)
    rng = np.random.default_rng(d + R)
    pages = 9
    n = pages * page
    c, keys, values = filled(rng, [n, n], 2, d, page, extra=0)
    assert c.table.shape[1] == pages
    q, q64 = bf16(rng, 2 * R, 4, d, scale=2.0)
    c.lens[0] = length or n + 1                    # one more than the row holds, too
    _check(c, q, q64, keys, values, R, d ** -0.5, [n, n], window=window)
    got = sph.kv_read(c, 0, R)
    for x, want in zip(got, (keys, values)):
        rows = np.zeros((2, R, 2, d))
        for s in range(2):
            rows[s] = want[s][n - R:]
        np.testing.assert_array_equal(host(x).reshape(2, R, 2, d), rows)
    # rows appended stand at the end of the row
    k, k64 = bf16(rng, 2 * R, 2, d)
    sph.kv_append(c, 0, k, k, R)
    c.lens[0] = n
    for x in sph.kv_read(c, 0, R):
        np.testing.assert_array_equal(host(x), O.quantize(k64))
    whole = sph.kv_read(c, 0, n)
    for x, want in zip(whole, (keys, values)):
        np.testing.assert_array_equal(host(x).reshape(2, n, 2, d)[:, :n - R], np.stack([w[:n - R] for w in want]))
