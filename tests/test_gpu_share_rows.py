"""Shared attention of calls with many rows on the GPU: rows taken from all over against the
64-bit oracle, each value within the bound of test_gpu_kv.py."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph
from oracle import kv_cache as O

from kv_build import bf16, host
from test_gpu_share import Text, ints, say

pytestmark = pytest.mark.gpu


def rows_are_right(t, q, out, lse, R, rows, window, picks):
    """Rows picks[s] of each session s, one at a time, as the last of what they see."""
    d, scale = t.d, t.d ** -0.5
    for s, mine in enumerate(picks):
        for r in mine:
            p = len(t.k[s]) - rows[s] + r
            at = s * R + r
            o, l = host(out[at]), host(lse[at])
            want, wl, mag, size = (x[0] for x in O.attend(host(q[at])[None], t.k[s][:p + 1], t.v[s][:p + 1], scale, 1, window))
            err = (d + 8) * 2.0 ** -24 * size
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -18 + 4 * err[..., None]) * mag + 1e-30
            assert (np.abs(o - want) <= tol).all(), (s, r, np.abs(o - want).max())
            tl = 2 * err + 2.0 ** -20 * np.maximum(1, np.abs(wl)) + (p + 65) * 2.0 ** -24
            assert (np.abs(l - wl) <= tl).all(), (s, r)


def shared_segments(plan):
    return int(host(plan.buffer)[:16].view(np.int32)[3])


# rows of all heads for which the parts' room holds 5, 4, 3 and 2 places: all three levels of what is
# shared, two, one
@pytest.mark.parametrize("R,levels", [(640, 3), (812, 3), (1000, 2), (1200, 1)])
@pytest.mark.parametrize("window", [0, 1500])
def test_fewer_levels_where_parts_would_take_too_much(R, levels, window):
    say("levels", R, levels, window)
    rng = np.random.default_rng(R)
    t = Text(rng, 5, 140, 400, 8, 256, 16)
    t.write([700, 0, 0, 0, 0])
    t.fork([0] * 4, [1, 2, 3, 4])
    t.write([650, 0, 0, 5, 7])
    t.fork([0, 0], [1, 2])
    t.write([620, 0, 30, 0, 0])
    t.fork([0], [1])
    rows = [33, 60, 20, 45, 3]
    t.write(rows)
    q, _ = bf16(rng, 5 * 60, 64, 256)
    q = torch.cat([torch.cat([x, x.new_zeros(R - 60, 64, 256)]) for x in q.split(60)])
    plan = sph.kv_share(t.c, 64, R, rows=ints(rows), window=window)
    places = (1 << 30) // (5 * R * 64 * (4 * 256 + 8))
    assert levels == min(3, places - 1) and plan.workspace_bytes <= (1 << 30) + 256
    if not window:
        assert shared_segments(plan) == levels
    out, lse = sph.kv_attend_shared(t.c, 0, q, plan, 256 ** -0.5, want_lse=True)
    rows_are_right(t, q, out, lse, R, rows, window, [sorted({0, n // 2, n - 1}) for n in rows])
    none = torch.cat([torch.arange(R, device="cuda") >= n for n in rows])
    assert (out[none] == 0).all() and torch.isneginf(lse[none]).all() and torch.isfinite(lse[~none]).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 90])
def test_rows_that_are_not_cut(d, window):
    # more than 65536 rows of a head: one shared level, no shares of a segment
    say("not cut", d, window)
    rng = np.random.default_rng(d)
    t = Text(rng, 3, 90, 220, 1, d, 16)
    t.write([640, 0, 0])
    t.fork([0, 0], [1, 2])
    rows = [700, 699, 650]
    t.write(rows)
    q, _ = bf16(rng, 3 * 700, 32, d)
    plan = sph.kv_share(t.c, 32, 700, rows=ints(rows), window=window)
    assert shared_segments(plan) == 1
    out, lse = sph.kv_attend_shared(t.c, 0, q, plan, d ** -0.5, want_lse=True)
    picks = [sorted({0, 1, 15, 16, n // 2, n - 2, n - 1} | set(rng.integers(0, n, 20).tolist())) for n in rows]
    rows_are_right(t, q, out, lse, 700, rows, window, picks)
