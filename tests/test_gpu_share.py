"""Attention of sessions with common pages on the GPU: against the 64-bit oracle, which
knows nothing of pages, within the bounds of test_gpu_kv.py, and against the plain call
on the same cache."""

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


class Text:
    """A cache of sessions and what each holds, one layer, as float64 [len, heads, d]."""

    def __init__(self, rng, n_slots, max_pages, n_pages, heads, d, page):
        self.rng, self.heads, self.d = rng, heads, d
        self.c = sph.KvCache.empty(1, n_pages, n_slots, max_pages, heads, d, page)
        self.c.pool.fill_(0xFF)  # scales that are no numbers
        self.k = [np.zeros((0, heads, d)) for _ in range(n_slots)]
        self.v = [np.zeros((0, heads, d)) for _ in range(n_slots)]

    def write(self, counts):
        """Each slot's next counts[slot] tokens."""
        R = max(max(counts), 1)
        assert host(sph.pages_grow(self.c, ints(counts))).tolist() == [0, 0]
        n = len(counts)
        k, k64 = bf16(self.rng, n * R, self.heads, self.d)
        v, v64 = bf16(self.rng, n * R, self.heads, self.d)
        sph.kv_append(self.c, 0, k, v, R, rows=ints(counts))
        for s, m in enumerate(counts):
            for held, x in ((self.k, k64), (self.v, v64)):
                held[s] = np.concatenate([held[s], O.quantize(x.reshape(n, R, self.heads, self.d)[s, :m])])

    def fork(self, parents, children):
        sph.pages_fork(self.c, ints(parents), ints(children))
        for p, c in zip(parents, children):
            self.k[c], self.v[c] = self.k[p], self.v[p]


def check(t, group, rows, window=0, slots=None, pad=0, max_len=0, seed=0, seen=None):
    """One call on the text's sessions against the oracle; returns (q, out, lse)."""
    rng = np.random.default_rng(seed)
    slots_of = list(range(len(rows))) if slots is None else slots
    n, R, d, Hq = len(rows), max(max(rows), 1), t.d, t.heads * group
    q, q64 = bf16(rng, n * R, Hq, d + pad)
    q, q64 = q[..., pad:], q64[..., pad:].reshape(n, R, Hq, d)
    scale = d ** -0.5
    r, sl = ints(rows), None if slots is None else ints(slots)
    plan = sph.kv_share(t.c, Hq, R, rows=r, slots=sl, window=window, max_len=max_len)
    out, lse = sph.kv_attend_shared(t.c, 0, q, plan, scale, want_lse=True)
    o, l = host(out).reshape(n, R, Hq, d), host(lse).reshape(n, R, Hq)
    for i, s in enumerate(slots_of):
        held = 0 <= s < len(t.k)
        k = t.k[s] if held else np.zeros((0, t.heads, d))
        v = t.v[s] if held else k
        want, wl, mag, size = O.attend(q64[i], k, v, scale, rows[i], window)
        err = (d + 8) * 2.0 ** -24 * size
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -18 + 4 * err[..., None]) * mag + 1e-30
        assert (np.abs(o[i] - want) <= tol).all(), (i, np.abs(o[i] - want).max())
        seen_rows = np.isfinite(wl)
        assert (l[i][~seen_rows] == -np.inf).all() and (o[i][~seen_rows] == 0).all()
        tl = 2 * err + 2.0 ** -20 * np.maximum(1, np.abs(wl)) + (len(k) + 64) * 2.0 ** -24
        assert (np.abs(l[i][seen_rows] - wl[seen_rows]) <= tl[seen_rows]).all()
    if seen is not None:
        head = host(plan.buffer)[:16].view(np.int32)
        assert (head[3] > 0) == seen, head  # segments that several sessions hold
    return q, out, lse, plan


SHAPES = [(1, 1, 64, 16), (2, 4, 128, 16), (8, 4, 128, 64), (3, 3, 64, 32), (2, 7, 256, 16), (4, 2, 256, 128), (1, 8, 64, 256),
          (2, 1, 128, 32)]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("rows", [1, 5, 9])
@pytest.mark.parametrize("window", [0, 100])
def test_branches_of_one_prompt(shape, rows, window):
    heads, group, d, page = SHAPES[shape]
    say("branches", SHAPES[shape], rows, window)
    t = Text(np.random.default_rng(shape), 6, 40 if page < 64 else 8, 400 if page < 64 else 60, heads, d, page)
    t.write([333, 0, 0, 0, 0, 0])
    t.fork([0] * 4, [1, 2, 3, 5])
    t.write([rows + 40, rows, rows + 3, rows + 100, rows, rows])  # slot 4 shares nothing
    check(t, group, [rows] * 6, window, seen=None if window else 333 // page * page * 4 >= 256)


def test_levels_of_groups():
    # trunk, documents, branches of branches: four levels of which three are shared
    t = Text(np.random.default_rng(20), 20, 64, 600, 2, 64, 16)
    t.write([100] + [0] * 19)
    t.fork([0] * 3, [1, 2, 3])
    t.write([170, 90, 200, 40] + [0] * 16)
    t.fork([0, 0, 0, 0, 1, 1, 2, 2, 2, 2, 2], [4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14])
    t.write([60] * 15 + [7] * 5)
    t.fork([4, 4, 12], [15, 16, 17])
    t.fork([15], [18])
    t.write([3] * 20)
    check(t, 4, [3] * 20, seen=True)
    check(t, 4, [1, 0, 3, 2] * 5, window=150, seen=None)
    # sessions in another order, some twice over pages but once each, some none
    check(t, 4, [3, 2, 3, 1, 3], slots=[14, 4, 16, 12, 15])
    check(t, 2, [3, 3, 3], slots=[-1, 4, 99])


def test_little_in_common_of_all_and_much_of_some():
    # one page of all three is worth no segment; two of them share 300 tokens more
    t = Text(np.random.default_rng(21), 4, 40, 120, 1, 64, 16)
    t.write([20, 0, 0, 0])
    t.fork([0, 0], [1, 2])
    t.write([310, 40, 0, 5])
    t.fork([0], [2])
    t.write([4, 4, 9, 4])
    check(t, 4, [3, 2, 3, 1], seen=True)
    check(t, 4, [3, 2, 3, 1], window=200)


@pytest.mark.parametrize("n", [1, 2, 3, 64, 65, 130])
def test_numbers_of_sessions(n):
    t = Text(np.random.default_rng(n), n, 24, 24 * n + 20, 1, 64, 16)
    t.write([130] + [0] * (n - 1))
    if n > 1:
        t.fork([0] * (n - 1), list(range(1, n)))
    t.write([1 + i % 7 for i in range(n)])
    check(t, 3, [1 + i % 2 for i in range(n)], seen=n > 1 if n * 128 >= 384 else None)


@pytest.mark.parametrize("d,page,long", [(64, 64, 9000), (128, 32, 7001), (256, 64, 5003)])
def test_long_documents_are_cut(d, page, long):
    # parts of one segment, and of sessions of very different lengths
    t = Text(np.random.default_rng(d), 5, long // page + 80, 2 * (long // page) + 250, 1, d, page)
    t.write([long, 0, 0, 0, 2000])
    t.fork([0, 0], [1, 2])
    t.write([5, 2500, 3, 4, 5])
    *_, plan = check(t, 4, [3, 3, 3, 3, 3], seen=True)
    assert host(plan.buffer)[:16].view(np.int32)[1] > 10  # items: more than segments and sessions
    check(t, 4, [3, 1, 2, 3, 3], window=1000)
    check(t, 4, [3] * 5, max_len=300, pad=8)  # any max_len
    check(t, 4, [3] * 5, pad=3)               # rows off 16 bytes


@pytest.mark.parametrize("d,page,rows", [(64, 16, 300), (128, 16, 200), (256, 32, 130)])
def test_prompts_behind_a_common_one(d, page, rows):
    t = Text(np.random.default_rng(rows), 3, 60, 200, 2, d, page)
    t.write([640, 0, 0])
    t.fork([0, 0], [1, 2])
    t.write([rows, rows - 7, 20])
    check(t, 2, [rows, rows - 7, 20], seen=True)
    check(t, 2, [rows, rows - 7, 20], window=64)
    # windows that begin inside what is common: those rows see part of it
    check(t, 2, [rows + 50, rows, 100])


@pytest.mark.parametrize("d,window", [(64, 0), (128, 0), (256, 0), (64, 90)])
def test_many_rows_are_not_cut(d, window):
    # more than 65536 rows of a head: one shared level, no shares of a segment; against the plain call
    t = Text(np.random.default_rng(d), 3, 90, 220, 1, d, 16)
    t.write([640, 0, 0])
    t.fork([0, 0], [1, 2])
    t.write([700, 699, 650])
    q, _ = bf16(np.random.default_rng(40), 3 * 700, 32, d)
    plan = sph.kv_share(t.c, 32, 700, rows=ints([700, 699, 650]), window=window)
    assert host(plan.buffer)[:16].view(np.int32)[3] == 1
    out, lse = sph.kv_attend_shared(t.c, 0, q, plan, d ** -0.5, want_lse=True)
    want, wl = sph.kv_attend(t.c, 0, q, 700, d ** -0.5, rows=ints([700, 699, 650]), window=window, want_lse=True)
    # both are within 2^-8 |o| + (2^-8 + 2^-18 + 4 s) sum |p v| of the exact outputs, |v| at most its largest
    most = max(np.abs(x).max() for x in t.v)
    assert (out.float() - want.float()).abs().max() <= 2 * (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -12) * most
    seen = torch.isfinite(wl)
    assert torch.equal(seen, torch.isfinite(lse)) and (lse[seen] - wl[seen]).abs().max() <= 1e-4


def test_rows_that_are_none_and_empty_slots():
    t = Text(np.random.default_rng(30), 6, 20, 60, 2, 128, 16)
    t.write([100, 0, 0, 0, 0, 0])
    t.fork([0, 0], [1, 2])
    t.write([2, 3, 0, 1, 0, 0])
    check(t, 2, [2, 3, 0, 4, 1, 0])      # more rows than tokens; slots 4, 5 are empty
    check(t, 2, [2, 3, 2, 1, 0, 0])      # rows of slot 2 lie on pages that it shares


def test_missing_pages_and_one_name_twice():
    # tables that the page calls do not make: a page that is none in what is shared, and the same page under two places
    t = Text(np.random.default_rng(31), 3, 20, 60, 1, 64, 16)
    t.write([200, 0, 0])
    t.fork([0, 0], [1, 2])
    t.write([20, 30, 40])
    t.c.table[:, 3] = -1
    t.c.table[1, 5] = t.c.table[1, 4]
    q, out, lse, _ = [None] * 4
    rng = np.random.default_rng(1)
    q, _ = bf16(rng, 3 * 2, 4, 64)
    plan = sph.kv_share(t.c, 4, 2)
    got = sph.kv_attend_shared(t.c, 0, q, plan, 0.125, want_lse=True)
    want = sph.kv_attend(t.c, 0, q, 2, 0.125, want_lse=True)
    assert torch.isfinite(got[0].float()).all()
    assert (got[0].float() - want[0].float()).abs().max() <= 2.0 ** -7 * want[0].float().abs().max()
    assert (got[1] - want[1]).abs().max() <= 1e-5


def test_no_number_stays_with_the_rows_that_see_it():
    t = Text(np.random.default_rng(32), 4, 20, 80, 1, 64, 16)
    t.write([64, 0, 0, 0])
    t.fork([0, 0], [1, 2])
    t.write([5, 5, 5, 70])
    k = torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda")
    k[2] = float("nan")
    assert host(sph.pages_grow(t.c, ints([1, 1, 1, 1]))).tolist() == [0, 0]
    sph.kv_append(t.c, 0, k, k, 1)
    q, _ = bf16(np.random.default_rng(2), 4 * 2, 2, 64)
    out, lse = sph.kv_attend_shared(t.c, 0, q, sph.kv_share(t.c, 2, 2), 0.125, want_lse=True)
    bad = torch.isnan(lse).any(-1).cpu().numpy().reshape(4, 2)
    assert bad.tolist() == [[False, False], [False, False], [False, True], [False, False]]
    assert np.isnan(host(out).reshape(4, 2, -1)[2, 1]).all() and np.isfinite(np.delete(host(out).reshape(8, -1), 5, 0)).all()


def test_a_plan_of_other_sizes_answers_nan():
    t = Text(np.random.default_rng(33), 2, 8, 20, 1, 64, 16)
    t.write([20, 30])
    plan, other = sph.kv_share(t.c, 2, 2), sph.kv_share(t.c, 2, 2, window=5)
    q, _ = bf16(np.random.default_rng(3), 4, 2, 64)
    plan.buffer.copy_(other.buffer[:plan.buffer.numel()])
    out, lse = sph.kv_attend_shared(t.c, 0, q, plan, 0.125, want_lse=True)
    assert torch.isnan(out.float()).all() and torch.isnan(lse).all()


def test_steps_captured_and_replayed():
    # plan, layers and growth in one graph; sessions grow from replay to replay
    rng = np.random.default_rng(34)
    c = sph.KvCache.empty(2, 200, 8, 24, 2, 128, 16)
    c.pool.random_(0, 256, generator=None)
    c.pool.view(2, 200, -1)[..., :] = 0x11  # finite scales and codes
    c.lens[0] = 0
    add = ints([1] * 8)
    sph.pages_grow(c, ints([200] + [0] * 7))
    sph.pages_fork(c, ints([0] * 6), ints([1, 2, 3, 4, 5, 6]))
    q = torch.zeros(8, 8, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(8, 2, 128, dtype=torch.bfloat16, device="cuda")
    plan = sph.kv_share(c, 8, 1)
    out = [torch.empty_like(q) for _ in range(2)]
    lse = [torch.empty(8, 8, device="cuda") for _ in range(2)]
    ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device="cuda")
    grow = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    status = torch.empty(2, dtype=torch.int32, device="cuda")

    def step():
        sph.pages_grow(c, add, workspace=grow, out=status)
        sph.kv_share(c, 8, 1, out=plan)
        for i in range(2):
            sph.kv_append(c, i, k, k, 1)
            sph.kv_attend_shared(c, i, q, plan, 0.1, workspace=ws, out=(out[i], lse[i]))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        q.copy_(bf16(rng, 8, 8, 128)[0])
        k.copy_(bf16(rng, 8, 2, 128)[0])
        graph.replay()
        torch.cuda.synchronize()
        assert host(status).tolist() == [0, 0]
        eager = sph.kv_share(c, 8, 1)
        for i in range(2):
            o, l = sph.kv_attend_shared(c, i, q, eager, 0.1, want_lse=True)
            assert torch.equal(o, out[i]) and torch.equal(l, lse[i])
            want, wl = sph.kv_attend(c, i, q, 1, 0.1, want_lse=True)
            assert (o.float() - want.float()).abs().max() <= 2.0 ** -6 * want.float().abs().max()
            assert (l - wl).abs().max() < 1e-4
