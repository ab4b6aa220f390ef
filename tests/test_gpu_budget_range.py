"""Shared attention, token weights and eviction at the ends of their ranges: pages beyond
32 bits of bytes, lengths that the table cannot name, values that are no numbers, thousands of
sessions, streams side by side.  What is compared with a call on another layout of the
same cache has to be equal bit for bit: neither place nor stream enters an order of sums."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph

from kv_build import bf16, host
from test_gpu_share import Text, check, ints, say

pytestmark = pytest.mark.gpu


def branches(seed, d, page=16, heads=2):
    t = Text(np.random.default_rng(seed), 5, 60, 200, heads, d, page)
    t.write([333, 0, 0, 0, 70])
    t.fork([0, 0, 0], [1, 2, 3])
    t.write([40, 5, 130, 5, 5])
    return t


def elsewhere(c, gap):
    """The same cache with pages `gap` bytes apart."""
    pool = torch.empty((c.layers, c.n_pages, gap), dtype=torch.uint8, device="cuda")[:, :, :c.pool.shape[2]]
    pool.copy_(c.pool)
    return sph.KvCache(pool, c.table.clone(), c.lens.clone(), c.refs.clone(), c.kv_heads, c.head_dim, c.page_tokens)


def attend_shared(c, q, R, scale=0.1, **kw):
    return sph.kv_attend_shared(c, 0, q, sph.kv_share(c, q.shape[1], R, n_sessions=q.shape[0] // R, **kw), scale, want_lse=True)


def same(x, y):
    assert all(torch.equal(a, b) for a, b in zip(x, y))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_pages_beyond_32_bits(d):
    c = branches(1, d).c
    far = elsewhere(c, 3 << 26)  # 200 pages of 192 MiB: 40 GB
    assert far.pool.stride(1) * (c.n_pages - 1) > 1 << 35
    q, _ = bf16(np.random.default_rng(2), 5 * 5, 4, d)
    out = attend_shared(c, q, 5)
    same(out, attend_shared(far, q, 5))
    n = c.table.shape[1] * 16
    w, v = torch.zeros(5, n, device="cuda"), torch.zeros(5, n, device="cuda")
    sph.kv_weigh(c, 0, q, out[1], 5, 0.1, w)
    sph.kv_weigh(far, 0, q, out[1], 5, 0.1, v)
    assert torch.equal(w, v) and float(w.sum()) > 0
    keep = ints([350, 330, 380, 335, 30])
    got = [sph.pages_evict(x, y, keep, 2, 5, want_kept=True) for x, y in ((c, w), (far, v))]
    same(*got)
    for name in ("table", "lens", "refs", "pool"):
        assert torch.equal(getattr(c, name), getattr(far, name)), name


@pytest.mark.parametrize("window", [0, 50])
def test_lengths_beyond_the_table(window):
    # what a slot's row cannot name is cut off, what is negative is none
    t = branches(3, 64)
    c = t.c
    most = c.table.shape[1] * 16
    c.table.clamp_(min=0)  # all places name a page; sessions share those that they held before
    c.pool.fill_(0x22)
    cut = elsewhere(c, c.pool.shape[2])
    c.lens.copy_(ints([most + 7, -3, 373, 2 ** 31 - 1, -2 ** 31]))
    cut.lens.copy_(ints([most, 0, 373, most, 0]))
    q, _ = bf16(np.random.default_rng(4), 5 * 2, 2, 64)
    out, want = attend_shared(c, q, 2, window=window), attend_shared(cut, q, 2, window=window)
    same(out, want)
    assert torch.isneginf(out[1].view(5, -1)[[1, 4]]).all() and torch.isfinite(out[1].view(5, -1)[[0, 2, 3]]).all()
    w, v = torch.zeros(5, most, device="cuda"), torch.zeros(5, most, device="cuda")
    sph.kv_weigh(c, 0, q, out[1], 2, 0.1, w, window=window)
    sph.kv_weigh(cut, 0, q, out[1], 2, 0.1, v, window=window)
    assert torch.equal(w, v) and (w[[1, 4]] == 0).all()
    for x in (c, cut):
        x.refs.fill_(1)  # (pages are named more than once here: as if each were of one slot)
    keep = ints([100, 5, 30, 40, 5])
    same(sph.pages_evict(c, w, keep, want_kept=True), sph.pages_evict(cut, v, keep, want_kept=True))
    assert host(c.lens).tolist() == [100, -3, 30, 40, -2 ** 31] and host(cut.lens).tolist() == [100, 0, 30, 40, 0]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 20, 32])
def test_values_that_are_no_number_by_rows_that_see_them(d, window):
    # token 48 of a common prompt; windows of some rows begin behind it
    t = Text(np.random.default_rng(5), 4, 40, 80, 1, d, 16)
    t.write([48, 0, 0, 0])
    k = torch.zeros(4, 1, d, dtype=torch.bfloat16, device="cuda")
    one = ints([1, 0, 0, 0])
    sph.pages_grow(t.c, one)
    sph.kv_append(t.c, 0, k, torch.full_like(k, float("nan")), 1, rows=one)
    t.write([15, 0, 0, 0])
    t.fork([0, 0], [1, 2])
    t.write([1, 5, 2, 7])
    assert host(t.c.lens).tolist() == [65, 69, 66, 7]
    q, _ = bf16(np.random.default_rng(6), 4 * 2, 2, d)
    out, lse = attend_shared(t.c, q, 2, window=window)
    sees = torch.tensor([s < 3 and (window == 0 or p - window < 48) for s, n in enumerate([65, 69, 66, 7]) for p in (n - 2, n - 1)])
    bad = torch.isnan(out.float()).flatten(1).cpu()
    assert (bad == sees[:, None]).all()
    assert (torch.isnan(lse).cpu() == sees[:, None]).all()  # (a token with such a value is held with keys that are none)


@pytest.mark.parametrize("n", [300, 600, 2048])
def test_thousands_of_sessions(n):
    # branches of eight prompts, in an order that mixes them; more than 256 are sorted in another way
    say("sessions", n)
    rng = np.random.default_rng(n)
    t = Text(rng, n, 20, 40 * 8 + 4 * n, 1, 64, 16)
    t.write([100 + 16 * i for i in range(8)] + [0] * (n - 8))
    t.fork([i % 8 for i in range(n - 8)], list(range(8, n)))
    t.write([1 + i % 5 for i in range(n)])
    order = rng.permutation(n).tolist()
    check(t, 2, [1] * n, slots=order, seen=True)
    check(t, 2, [1 + i % 2 for i in range(n)], slots=order, window=70)


@pytest.mark.parametrize("n", [3, 20, 70])
@pytest.mark.parametrize("places", [1, 2, 3, 4, 5, 7])
def test_rows_of_few_places(places, n):
    # tables of as many pages as the longest slot holds, the last row of them at the end of its memory
    t = Text(np.random.default_rng(places), n, places, places * n + 4, 1, 64, 64)
    t.write([max(64 * (places - 1), 40)] + [0] * (n - 1))
    t.fork([0] * (n - 1), list(range(1, n)))
    t.write([1 + i % 20 for i in range(n)])
    *_, plan = check(t, 2, [1 + i % 2 for i in range(n)])
    assert host(plan.buffer)[:16].view(np.int32)[3] == (64 * (places - 1) * (n - 1) >= 256)


def test_what_is_not_worth_a_part_is_left_to_the_sessions():
    # 32 tokens in common of 40 sessions with 40 rows each: read beside each session's own
    t = Text(np.random.default_rng(11), 40, 8, 200, 1, 64, 16)
    t.write([32] + [0] * 39)
    t.fork([0] * 39, list(range(1, 40)))
    t.write([5 + i % 9 for i in range(40)])
    check(t, 8, [5] * 40, seen=False)


@pytest.mark.parametrize("n", [4, 40, 100])
def test_rows_differ_at_any_place(n):
    # sessions leave their prompt at places all along its 600 pages, some but at the last
    rng = np.random.default_rng(n)
    t = Text(rng, n, 620, 620 * 3 + 3 * n, 1, 64, 16)
    t.write([9601] + [0] * (n - 1))
    t.fork([0] * (n - 1), list(range(1, n)))
    t.write([1 + i % 3 for i in range(n)])
    base = host(t.c.table)
    table, other = base.copy(), base[0].copy()
    other[:600] = np.setdiff1d(np.arange(t.c.n_pages), base)[:600]
    t.c.pool[:, other[:600]] = t.c.pool[:, base[0, :600]]  # the same text on pages of its own
    at = np.unique(np.concatenate([rng.integers(0, 600, n - 1), [599, 3, 255, 256]]))[-(n - 1):]
    for s in range(1, n):
        p = at[s % len(at)]
        table[s, p:600] = other[p:600]
    t.c.table.copy_(torch.from_numpy(table))
    check(t, 1, [1] * n, seen=True)


def test_weights_and_eviction_of_many_slots():
    n = 3000
    t = Text(np.random.default_rng(7), n, 6, 4 * n, 1, 64, 16)
    t.write([1 + i % 40 for i in range(n)])
    q, _ = bf16(np.random.default_rng(8), n, 2, 64)
    out, lse = sph.kv_attend(t.c, 0, q, 1, 0.1, want_lse=True)
    w = torch.zeros(n, 96, device="cuda")
    sph.kv_weigh(t.c, 0, q, lse, 1, 0.1, w)
    # each of the two heads gives one away: a weight is off by 2^-20 and 76 2^-24 (1 + size + |lse|), these at most 13
    # together, and its log-sum-exp by no more
    assert (w.double().sum(1) - 2).abs().max() <= 2 * (2.0 ** -20 + 2 * 76 * 14 * 2.0 ** -24)
    lens = host(t.c.lens)
    keep = np.asarray([1 + i % 23 for i in range(n)])
    before = host(w)
    _, kept = sph.pages_evict(t.c, w, ints(keep), want_kept=True)
    left = np.minimum(lens, keep)
    np.testing.assert_array_equal(host(t.c.lens), left)
    assert int(t.c.refs.sum()) == int((-(-left // 16)).sum()) == int((t.c.table >= 0).sum())
    kept, after = host(kept), host(w)
    for s in range(0, n, 37):
        np.testing.assert_array_equal(after[s, :left[s]], before[s, kept[s, :left[s]]])
        dropped = np.setdiff1d(np.arange(lens[s]), kept[s, :left[s]])
        assert len(dropped) == 0 or before[s, dropped].max() <= after[s, :left[s]].min()


def test_streams_side_by_side():
    # calls with plans and workspaces of their own, on one cache, from two streams
    c = branches(9, 128).c
    q = [bf16(np.random.default_rng(10 + i), 5 * 3, 8, 128)[0] for i in range(2)]
    want = [attend_shared(c, x, 3) for x in q]
    n = c.table.shape[1] * 16
    sums = [sph.kv_weigh(c, 0, x, y[1], 3, 0.1, torch.zeros(5, n, device="cuda")) for x, y in zip(q, want)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in q]
    got = [[], []]
    for _ in range(8):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                out = attend_shared(c, q[i], 3)
                got[i].append((*out, sph.kv_weigh(c, 0, q[i], out[1], 3, 0.1, torch.zeros(5, n, device="cuda"))))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            same(g, (*want[i], sums[i]))
