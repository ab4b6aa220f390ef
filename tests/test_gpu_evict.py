"""Eviction on the GPU against the oracle's lists, exactly: what every slot keeps, in
every layer and head, and that nothing else changes."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph
from oracle import kv_budget as O

from kv_build import host, tables

pytestmark = pytest.mark.gpu


def say(*a):
    print("[gpu]", *a, flush=True)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def cache_of(rng, lens, heads, d, page, layers, **kw):
    """A cache of random bytes with pages in random order."""
    table, refs = tables(rng, lens, page, **kw)
    pool = torch.from_numpy(rng.integers(0, 256, (layers, len(refs), sph.kv_page_bytes(heads, d, page)), dtype=np.uint8)).cuda()
    full = np.zeros(len(table), np.int32)
    full[:len(lens)] = lens
    return sph.KvCache(pool, torch.from_numpy(table).cuda(), torch.from_numpy(full).cuda(),
                       torch.from_numpy(refs).cuda(), heads, d, page)


def token_bytes(pages, heads, d, page):
    """[layers, pages, tokens, heads, 17 d / 16]: each token's bytes of its page."""
    L, P, _ = pages.shape
    b = pages.reshape(L, P, heads, page // 16, 17 * d)
    k = b[..., :8 * d].reshape(L, P, heads, page // 16, 16, d // 2)
    v = b[..., 8 * d:16 * d].reshape(L, P, heads, page // 16, 4, 16, 4, d // 32)
    v = np.swapaxes(v, -3, -2).reshape(L, P, heads, page // 16, 16, d // 2)
    ks, vs = [np.swapaxes(b[..., a:a + d // 2].reshape(L, P, heads, page // 16, d // 32, 16), -1, -2)
              for a in (16 * d, 16 * d + d // 2)]
    t = np.concatenate([k, v, ks, vs], -1).reshape(L, P, heads, page, -1)
    return np.swapaxes(t, 2, 3)


def look(c):
    return {n: host(t).copy() for n, t in (("pool", c.pool), ("table", c.table), ("lens", c.lens), ("refs", c.refs))}


def check(c, was, weights, keep, first, recent, w_out, kept, w_before):
    """Everything after an eviction against the oracle's choice on what was before."""
    page, heads, d = c.page_tokens, c.kv_heads, c.head_dim
    want, table, lens, refs = O.evict(was["table"], was["lens"], was["refs"], weights, keep, first, recent, page)
    np.testing.assert_array_equal(host(c.lens), lens)
    np.testing.assert_array_equal(host(c.table), table)
    np.testing.assert_array_equal(host(c.refs), refs)
    nb = sph.kv_page_bytes(heads, d, page)
    now, old = host(c.pool), was["pool"]
    np.testing.assert_array_equal(now[:, :, nb:], old[:, :, nb:])
    old_t = token_bytes(old[:, :, :nb], heads, d, page)
    expect = old_t.copy()
    for s, k in enumerate(want):
        k = np.asarray(k, np.int64)
        i = np.arange(len(k))
        expect[:, was["table"][s, i // page], i % page] = old_t[:, was["table"][s, k // page], k % page]
        n = int(was["lens"][s])
        np.testing.assert_array_equal(w_out[s, :len(k)], weights[s, k])
        assert not w_out[s, len(k):n].any()
        np.testing.assert_array_equal(w_out[s, n:], w_before[s, n:])
        if kept is not None:
            np.testing.assert_array_equal(kept[s, :len(k)], k)
            assert (kept[s, len(k):] == -1).all()
    np.testing.assert_array_equal(token_bytes(now[:, :, :nb], heads, d, page), expect)


def weights_of(rng, slots, width, kind):
    w = np.exp(2 * rng.standard_normal((slots, width))).astype(np.float32)
    if kind == "ties":
        w = np.round(w * 2).astype(np.float32) / 2
    elif kind == "equal":
        w[:] = 0.5
    elif kind == "odd":  # signs, zeros of both, infinities, NaN of both, subnormals, the largest
        some = np.array([0.0, -0.0, np.inf, -np.inf, np.nan, -np.nan, 1e-45, -1e-45, 3.4028235e38, -3.4028235e38, 1.0, -1.0],
                        np.float32)
        w = some[rng.integers(0, len(some), (slots, width))]
    return w


CASES = [  # heads, d, page, layers, lens, keep, first, recent, weights
    (1, 64, 16, 1, [1], [0], 0, 0, "random"),
    (1, 128, 16, 1, [1], [1], 0, 0, "random"),
    (2, 64, 16, 2, [0, 1, 15, 16, 17, 33], [0, 0, 7, 15, 16, 2], 0, 0, "random"),
    (3, 128, 32, 2, [40, 64, 65, 300], [39, 1, 64, 150], 4, 8, "random"),
    (2, 256, 64, 3, [200, 64, 63, 129, 1], [100, 63, 1, 128, 5], 1, 1, "ties"),
    (1, 256, 16, 1, [500], [499], 0, 0, "ties"),
    (5, 64, 128, 2, [1000, 517, 128], [-5, 516, 127], 3, 2, "equal"),
    (1, 128, 256, 1, [4095, 4096, 4097], [2048, 4095, 1], 0, 300, "odd"),
    (2, 64, 16, 1, [9000, 8193], [5000, 100], 16, 64, "odd"),
    (1, 128, 64, 2, [5000, 3, 700], [2500, 3, 10000], 5000, 0, "random"),
    (1, 128, 64, 1, [1000, 1000], [10, 900], 20, 1 << 40, "random"),
    (4, 128, 16, 2, [777] * 9, [776, 775, 700, 400, 100, 16, 1, 0, 777], 0, 0, "ties"),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("apart", [False, True])
def test_keeps_the_largest(case, apart):
    heads, d, page, layers, lens, keep, first, recent, kind = CASES[case]
    rng = np.random.default_rng(case)
    c = cache_of(rng, lens, heads, d, page, layers, n_slots=len(lens) + 1)
    width = c.table.shape[1] * page
    # (rows further apart than they need be)
    w = weights_of(rng, len(lens) + 1, width + 24, kind)
    weights = torch.from_numpy(w).cuda()[:, 8:8 + width]
    say("evict", CASES[case][:4], lens, "apart" if apart else "in place")
    was, keep = look(c), keep + [3]
    if apart:
        out = torch.full_like(weights, 7.0), torch.full((len(lens) + 1, width + 3), -1, dtype=torch.int32, device="cuda")
        got = sph.pages_evict(c, weights, ints(keep), first, recent, out=out)
        assert got[0] is out[0] and got[1] is out[1]
        np.testing.assert_array_equal(host(weights), host(torch.from_numpy(w[:, 8:8 + width])))
        check(c, was, w[:, 8:8 + width], keep, first, recent, host(out[0]), host(out[1]), np.full((len(w), width), 7.0))
    else:
        got = sph.pages_evict(c, weights, ints(keep), first, recent, want_kept=True)
        assert got[0] is weights
        check(c, was, w[:, 8:8 + width], keep, first, recent, host(weights), host(got[1]), w[:, 8:8 + width])


@pytest.mark.parametrize("page,trunk,own", [(16, 100, 200), (64, 64, 70), (32, 33, 500)])
def test_shared_pages_stay(page, trunk, own):
    # four slots share their first pages; what they share is kept and moves nowhere
    rng = np.random.default_rng(page)
    c = cache_of(rng, [trunk], 2, 64, page, 2, n_slots=6, n_pages=400, extra=own // page + 2)
    sph.pages_fork(c, ints([0, 0, 0]), ints([1, 2, 4]))
    sph.pages_grow(c, ints([own, own // 2, 3, 0, own, 0]))
    was = look(c)
    width = c.table.shape[1] * page
    w = weights_of(rng, 6, width, "random")
    keep = [trunk + 10, trunk // 2, 0, 5, trunk + own - 1, 0]
    weights = torch.from_numpy(w).cuda()
    sph.pages_evict(c, weights, ints(keep), 2, 5)
    check(c, was, w, keep, 2, 5, host(weights), None, w)
    # a session that shares its half-filled last page keeps all of it
    sph.pages_fork(c, ints([0]), ints([5]))
    was, w = look(c), host(weights).astype(np.float32)
    sph.pages_evict(c, weights, ints([0] * 6), 0, 0)
    check(c, was, w, [0] * 6, 0, 0, host(weights), None, w)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32), (256, 16)])
def test_many_layers_and_slots(d, page):
    # 4160 units of a slot, layer and head: workgroups of two waves
    rng = np.random.default_rng(d)
    lens = [int(n) for n in rng.integers(0, 150, 65)]
    c = cache_of(rng, lens, 2, d, page, 32)
    assert c.n_slots * c.layers * c.kv_heads >= 4096
    was = look(c)
    w = weights_of(rng, 65, c.table.shape[1] * page, "ties")
    weights = torch.from_numpy(w).cuda()
    keep = [int(n) for n in rng.integers(0, 150, 65)]
    sph.pages_evict(c, weights, ints(keep), 3, 9)
    check(c, was, w, keep, 3, 9, host(weights), None, w)


@pytest.mark.parametrize("n", [4096, 4097, 8192, 8193, 16384, 16385, 40000])
def test_long_slots(n):
    # weights in registers up to 4096, 8192 and 16384 tokens, read again beyond
    rng = np.random.default_rng(n)
    c = cache_of(rng, [n, 5], 1, 64, 256, 1)
    for kind, keep in (("odd", n // 2), ("random", n // 3), ("equal", n // 4)):
        was = look(c)
        w = weights_of(rng, 2, c.table.shape[1] * 256, kind)
        weights = torch.from_numpy(w).cuda()
        _, kept = sph.pages_evict(c, weights, ints([keep, 2]), 1, 100, want_kept=True)
        check(c, was, w, [keep, 2], 1, 100, host(weights), host(kept), w)


def test_every_slot_emptied_and_filled_again():
    rng = np.random.default_rng(5)
    c = cache_of(rng, [100, 50, 7], 1, 128, 16, 2)
    weights = torch.rand(3, c.table.shape[1] * 16, device="cuda")
    sph.pages_evict(c, weights, ints([0, 0, 0]))
    assert not host(c.lens).any() and not host(c.refs).any() and (host(c.table) == -1).all()
    assert host(sph.pages_grow(c, ints([100, 1, 0]))).tolist() == [0, 0]


def test_missing_pages():
    # a token whose page is none moves as zeros, one whose place is on no page goes nowhere
    rng = np.random.default_rng(6)
    c = cache_of(rng, [200], 1, 64, 16, 1)
    c.table[0, 3] = -1
    c.table[0, 9] = 1 << 20
    before = look(c)
    width = c.table.shape[1] * 16
    w = np.arange(width, dtype=np.float32)[None] % 7
    weights = torch.from_numpy(w).cuda()
    _, kept = sph.pages_evict(c, weights, ints([120]), want_kept=True)
    want = O.choose(w[0], 200, 120, 0, 0)
    np.testing.assert_array_equal(host(kept)[0, :120], want)
    old = token_bytes(before["pool"], 1, 64, 16)
    new = token_bytes(host(c.pool), 1, 64, 16)
    live = set(range(old.shape[1]))
    for i, j in enumerate(want):
        at, src = before["table"][0, i // 16], before["table"][0, j // 16]
        if at not in live:
            continue
        expect = old[0, src, j % 16] if src in live else np.zeros_like(old[0, 0, 0])
        np.testing.assert_array_equal(new[0, at, i % 16], expect)


def test_long_row_and_page_stride():
    # pages further apart than they need be, and layers too
    rng = np.random.default_rng(7)
    table, refs = tables(rng, [600, 300], 32)
    nb = sph.kv_page_bytes(2, 64, 32)
    big = torch.from_numpy(rng.integers(0, 256, (3, len(refs) + 2, nb + 48), dtype=np.uint8)).cuda()
    pool = big[:2, 1:-1]
    c = sph.KvCache(pool, ints(table), ints([600, 300]), ints(refs), 2, 64, 32)
    was = look(c)
    edge = host(big).copy()
    w = weights_of(rng, 2, table.shape[1] * 32, "random")
    weights = torch.from_numpy(w).cuda()
    sph.pages_evict(c, weights, ints([301, 100]), 1, 7)
    check(c, was, w, [301, 100], 1, 7, host(weights), None, w)
    now = host(big)
    np.testing.assert_array_equal(now[2], edge[2])
    np.testing.assert_array_equal(now[:, [0, -1]], edge[:, [0, -1]])


def test_captured_and_replayed():
    rng = np.random.default_rng(8)
    lens = [300, 170, 33, 1]
    c = cache_of(rng, lens, 2, 128, 16, 2, n_pages=80)
    width = c.table.shape[1] * 16
    weights = torch.zeros(4, width, device="cuda")
    after, kept = torch.zeros_like(weights), torch.full((4, width), -1, dtype=torch.int32, device="cuda")
    keep = ints([200, 100, 20, 1])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sph.pages_evict(c, weights, ints([300, 170, 33, 1]), out=(after, kept))  # nothing to drop
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sph.pages_evict(c, weights, keep, 1, 3, out=(after, kept))
    for turn in range(4):
        torch.cuda.synchronize()
        now = host(c.lens)
        status = sph.pages_grow(c, ints(np.asarray(lens) - now))
        assert host(status).tolist() == [0, 0]
        w = weights_of(rng, 4, width, ("random", "ties", "odd", "equal")[turn])
        weights.copy_(torch.from_numpy(w))
        after.fill_(7.0)
        kept.fill_(-1)
        was = look(c)
        graph.replay()
        torch.cuda.synchronize()
        check(c, was, w, [200, 100, 20, 1], 1, 3, host(after), host(kept), np.full((4, width), 7.0))


def test_two_streams_of_their_own():
    rng = np.random.default_rng(9)
    both = [cache_of(rng, [2000, 900], 2, 64, 16, 2) for _ in range(2)]
    ws = [weights_of(rng, 2, c.table.shape[1] * 16, "random") for c in both]
    was = [look(c) for c in both]
    t = [torch.from_numpy(w).cuda() for w in ws]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    keep = ints([1000, 400])
    torch.cuda.synchronize()
    for c, w, s in zip(both, t, streams):
        with torch.cuda.stream(s):
            sph.pages_evict(c, w, keep, 0, 10)
    torch.cuda.synchronize()
    for c, w, w0, a in zip(both, t, ws, was):
        check(c, a, w0, [1000, 400], 0, 10, host(w), None, w0)
