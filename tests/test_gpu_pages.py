"""Page upkeep on the GPU against the oracle's lists, exactly: tables, lengths,
counts and what every page holds."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph
from oracle import kv_cache as O

from kv_build import bf16, host

pytestmark = pytest.mark.gpu


def say(*a):
    print("[gpu]", *a, flush=True)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


class Both:
    """A cache and the oracle's, with pages that hold their first number in every byte."""

    def __init__(self, n_pages, n_slots, max_pages, page, layers=2, heads=1, d=64, seed=0):
        self.o = O.Pages(n_pages, n_slots, max_pages, page)
        self.c = sph.KvCache.empty(layers, n_pages, n_slots, max_pages, heads, d, page)
        stamp = torch.arange(n_pages, dtype=torch.int32, device="cuda").view(1, -1, 1) * 7 + \
            torch.arange(layers, device="cuda", dtype=torch.int32).view(-1, 1, 1) * 1000003
        self.words = self.c.pool.view(torch.int32)
        self.words.copy_(stamp.expand_as(self.words))
        self.words += torch.arange(self.words.shape[2], dtype=torch.int32, device="cuda") * 131
        self.fresh = self.words.clone()

    def same(self):
        np.testing.assert_array_equal(host(self.c.lens), self.o.lens)
        np.testing.assert_array_equal(host(self.c.refs), self.o.refs)
        np.testing.assert_array_equal(host(self.c.table), self.o.table)
        want = self.fresh[:, torch.tensor(self.o.content).cuda()]
        live = torch.tensor(np.flatnonzero(self.o.refs > 0)).cuda()
        assert torch.equal(self.words[:, live], want[:, live])

    def grow(self, add):
        status = sph.pages_grow(self.c, ints(add))
        assert tuple(host(status).tolist()) == self.o.grow(np.asarray(add))

    def trim(self, kept):
        sph.pages_trim(self.c, ints(kept))
        self.o.trim(kept)

    def fork(self, parents, children):
        sph.pages_fork(self.c, ints(parents), ints(children))
        self.o.fork(parents, children)

    def compact(self, apart=False):
        out = (torch.full_like(self.c.table, -7), torch.full_like(self.c.refs, -7)) if apart else None
        table, refs, live = sph.pages_compact(self.c, out=out)
        assert int(live) == self.o.compact()
        if apart:
            self.c.table.copy_(table)
            self.c.refs.copy_(refs)


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n_pages,n_slots,max_pages,layers,heads", [
    (40, 5, 9, 1, 1), (300, 17, 40, 3, 2), (5000, 40, 200, 2, 1), (9000, 3, 4000, 1, 1),
    # past what one workgroup takes: pages, slots
    (140000, 6, 30000, 1, 1), (6000, 4500, 5, 1, 1),
])
def test_random_walk(n_pages, n_slots, max_pages, layers, heads, page):
    rng = np.random.default_rng(n_pages + page)
    b = Both(n_pages, n_slots, max_pages, page, layers, heads)
    b.same()
    for step in range(12):
        what = ["grow", "grow", "trim", "fork", "grow", "compact"][step % 6]
        say("walk", n_pages, page, step, what)
        if what == "grow":
            most = max(1, min(n_pages * page // n_slots // 3, max_pages * page // 3))
            b.grow(rng.integers(-3, most, n_slots) * (rng.random(n_slots) < 0.8))
        elif what == "trim":
            b.trim([int(n * rng.random()) - 1 if rng.random() < 0.7 else int(n) + 5 for n in b.o.lens])
        elif what == "fork":
            order = rng.permutation(n_slots)
            k = n_slots // 2
            b.fork(order[:1].tolist() * k if step < 6 else order[:k].tolist(), order[k:2 * k].tolist())
        else:
            b.compact(apart=step > 6)
        b.same()


def test_growth_finds_pages_far_back():
    # free pages only at the end of the pool, as many as are needed
    for n_pages in (100, 20000, 131072, 131073):
        say("far back", n_pages)
        b = Both(n_pages, 3, n_pages, 16, layers=1)
        b.grow([(n_pages - 5) * 16, 0, 0])
        b.grow([0, 33, 32])
        b.same()
        b.grow([1, 0, 0])
        b.trim([0, 33, 32])
        b.grow([5, 5, 5])
        b.same()


def test_nothing_changes_when_it_does_not_fit():
    b = Both(10, 3, 6, 16)
    b.grow([40, 20, 0])
    b.same()
    say("too few pages")
    b.grow([80, 80, 1])          # lacking pages, and a row too short
    b.grow([0, 0, 90])
    b.grow([0, 70, 0])
    b.same()
    b.grow([8, 0, 80])           # five pages
    b.grow([16, 0, 0])           # the last one
    b.same()
    assert (b.o.refs > 0).all()
    say("full pool")
    b.grow([0, 0, 0])
    b.compact()
    b.same()
    b.grow([1, 0, 0])
    b.same()


def test_every_holder_of_a_page_grows():
    # four slots share a partly filled page: each gets its own copy, the page is free
    b = Both(64, 5, 8, 32, layers=4, heads=3, d=128)
    b.grow([70, 0, 0, 0, 10])
    b.fork([0, 0, 0], [1, 2, 3])
    b.same()
    b.grow([1, 33, 0, 5, 0])
    b.same()
    b.grow([0, 0, 9, 0, 0])      # the one left is alone: no copy
    b.same()


def test_full_pages_stay_shared_and_trimmed_ones_are_copied():
    b = Both(64, 3, 8, 16)
    b.grow([48, 0, 0])
    b.fork([0], [1])
    b.grow([5, 5, 0])            # the shared text ends with its page: nothing to copy
    b.same()
    b.trim([48, 40, 0])          # into a shared page
    b.grow([0, 3, 0])
    b.same()


def test_pairs_out_of_range_are_passed_over():
    b = Both(20, 3, 4, 16)
    b.grow([20, 10, 0])
    say("odd pairs")
    sph.pages_fork(b.c, ints([0, 0, 9]), ints([0, 3, 2]))
    sph.pages_fork(b.c, ints([-1, 1]), ints([2, -1]))
    sph.pages_copy(b.c, ints([0, 1, -1, 20, 2]), ints([20, -1, 5, 5, 2]))
    b.same()


def test_copy():
    b = Both(50, 2, 4, 64, layers=3, heads=2, d=128)
    src, dst = [3, 7, 7, 40], [10, 11, 12, 0]
    sph.pages_copy(b.c, ints(src), ints(dst))
    want = b.fresh.clone()
    want[:, dst] = b.fresh[:, src]
    assert torch.equal(b.words, want)


def test_strided_tables_and_pools():
    page, heads, d = 16, 1, 64
    nb = sph.kv_page_bytes(heads, d, page)
    wide = torch.full((4, 20), -9, dtype=torch.int32, device="cuda")
    wide[:, :6] = -1
    pool = torch.zeros((2, 30, nb + 48), dtype=torch.uint8, device="cuda")
    c = sph.KvCache(pool, wide[:, :6], torch.zeros(4, dtype=torch.int32, device="cuda"),
                    torch.zeros(30, dtype=torch.int32, device="cuda"), heads, d, page)
    o = O.Pages(30, 4, 6, page)
    for add in ([17, 3, 0, 90], [16, 0, 5, 1]):
        sph.pages_grow(c, ints(add))
        o.grow(np.asarray(add))
    sph.pages_trim(c, ints([5, 0, 5, 5]))
    o.trim([5, 0, 5, 5])
    table, refs, live = sph.pages_compact(c)
    assert int(live) == o.compact()
    np.testing.assert_array_equal(host(c.table), o.table)
    np.testing.assert_array_equal(host(c.refs), o.refs)
    assert bool((wide[:, 6:] == -9).all())


def test_a_step_in_a_graph():
    """Grow, append, attend and trim captured once and replayed, against the same calls."""
    rng = np.random.default_rng(5)
    n, R, heads, hq, d, page = 3, 4, 2, 8, 128, 16

    def start():
        c = sph.KvCache.empty(2, 80, n, 20, heads, d, page)
        sph.pages_grow(c, ints([37, 5, 200]))
        k, _ = bf16(np.random.default_rng(1), n * 200, heads, d)
        for layer in range(2):
            sph.kv_append(c, layer, k, k.flip(0), 200, rows=c.lens.clone())
        return c

    feeds = [[bf16(rng, n * R, h, d)[0] for h in (heads, heads, hq)] for _ in range(4)]
    keep = [ints(x) for x in ([2, 1, 4], [1, 1, 1], [4, 4, 4], [3, 1, 2])]
    add = ints([R] * n)

    def step(c, k, v, q, dropped, ws, grow_ws, out, status):
        sph.pages_grow(c, add, workspace=grow_ws, out=status)
        for layer in range(2):
            sph.kv_append(c, layer, k, v, R)
            sph.kv_attend(c, layer, q, R, 0.1, workspace=ws, out=(out[layer], None))
        sph.pages_trim(c, c.lens - R + dropped)

    def buffers(c):
        ws = torch.empty(max(sph.kv_attend_workspace(c, hq, n, R), 1), dtype=torch.uint8, device="cuda")
        grow_ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
        out = torch.zeros(2, n * R, hq, d, dtype=torch.bfloat16, device="cuda")
        return ws, grow_ws, out, torch.zeros(2, dtype=torch.int32, device="cuda")

    eager, graphed = start(), start()
    be, bg = buffers(eager), buffers(graphed)
    fixed = [x.clone() for x in feeds[0]] + [keep[0].clone()]
    torch.cuda.synchronize()
    say("capture")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graphed, *fixed, *bg)
    for feed, kept in zip(feeds, keep):
        for dst, src in zip(fixed, feed + [kept]):
            dst.copy_(src)
        step(eager, *feed, kept, *be)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(be[2], bg[2]) and bool(be[2].any())
        for name in ("table", "lens", "refs"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), name
        assert host(bg[3]).tolist() == [0, 0]
