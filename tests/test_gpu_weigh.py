"""Token weights on the GPU against the 64-bit oracle.

A score's products are exact in fp32 and their sums round, D + 8 times at most, so it is
within (D + 8) 2^-24 of its size (scale * sum |q k|); scaling it, the log-sum-exp in
fp32 and their difference round by 4 more 2^-24 of their sizes, and the exponential by
2^-20 (its own and the units it is taken in). `slack` is the sum of the terms, each
times 1 + size + |lse|. The sum of N terms rounds N 2^-24, and what was there once more:

    2^-24 (D + 12) slack + (2^-20 + N 2^-24) sum + 2^-24 |result|
"""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph
from oracle import kv_budget as B
from oracle import kv_cache as O

from kv_build import bf16, filled, host

pytestmark = pytest.mark.gpu


def say(*a):
    print("[gpu]", *a, flush=True)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def within(got, before, total, slack, d, terms):
    want = before + total
    tol = 2.0 ** -24 * (d + 12) * slack + (2.0 ** -20 + terms * 2.0 ** -24) * total + 2.0 ** -24 * np.abs(want)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])


CASES = [  # kv heads, group, d, page, lens, rows, window
    (1, 1, 64, 16, [1], [1], 0),
    (1, 1, 128, 16, [5], [1], 0),
    (2, 4, 128, 16, [40, 1, 300, 0], [1, 1, 1, 1], 0),
    (8, 4, 128, 64, [700, 515, 20], [5, 5, 5], 0),
    (3, 3, 64, 32, [513, 511, 512, 100], [9, 0, 4, 9], 0),
    (2, 7, 256, 16, [260, 255, 31], [6, 6, 3], 0),
    (1, 2, 128, 128, [200, 129], [100, 129], 0),
    (2, 1, 64, 16, [600, 77], [300, 77], 0),
    (2, 2, 128, 32, [700, 90], [5, 3], 64),
    (1, 3, 64, 16, [400, 300], [200, 17], 33),
    (1, 2, 256, 64, [300, 64], [64, 40], 1),
    (2, 2, 128, 16, [3, 2], [7, 2], 0),           # more rows than tokens: the first see nothing
    (4, 8, 64, 256, [1100], [8], 1000),
    (16, 1, 128, 16, [33], [33], 0),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("fresh", [False, True])
def test_sums_of_weights(case, fresh):
    heads, group, d, page, lens, rows, window = CASES[case]
    rng = np.random.default_rng(case)
    say("weigh", CASES[case], "fresh" if fresh else "")
    c, keys, _ = filled(rng, lens, heads, d, page, n_slots=len(lens) + 2)
    R, n = max(rows), len(lens)
    pad = 8 if case % 2 else 3  # with 3, rows of q are off 16 bytes
    q, q64 = bf16(rng, n * R, heads * group, d + pad)
    q, q64 = q[..., pad:], q64[..., pad:].reshape(n, R, heads * group, d)
    scale = d ** -0.5
    width = c.table.shape[1] * page
    w = rng.random((len(lens) + 2, width + 5)).astype(np.float32)
    weights = torch.from_numpy(w).cuda()
    lse = np.full((n, R, heads * group), -np.inf)
    sums = []
    for s in range(n):
        lse[s] = O.attend(q64[s], keys[s], keys[s], scale, rows[s], window)[1]
        sums.append(B.weigh(q64[s], keys[s], lse[s], scale, rows[s], window))
    lse32 = torch.from_numpy(lse.reshape(n * R, -1).astype(np.float32)).cuda()
    got = sph.kv_weigh(c, 0, q, lse32, R, scale, weights, rows=ints(rows), window=window, fresh=fresh)
    assert got is weights
    again = torch.from_numpy(w).cuda()
    sph.kv_weigh(c, 0, q, lse32, R, scale, again, rows=ints(rows), window=window, fresh=fresh, max_len=1)
    tight = torch.from_numpy(w).cuda()
    sph.kv_weigh(c, 0, q, lse32, R, scale, tight, rows=ints(rows), window=window, fresh=fresh, max_len=max(lens))
    for t in (weights, again, tight):  # any max_len
        g = host(t)
        for s in range(n):
            before = w[s, :lens[s]].astype(np.float64)
            if fresh:
                before[max(0, lens[s] - rows[s]):] = 0
            within(g[s, :lens[s]], before, *sums[s], d, R * heads * group)
            np.testing.assert_array_equal(g[s, lens[s]:], w[s, lens[s]:])
        np.testing.assert_array_equal(g[n:], w[n:])
    for s in range(n):  # each row gives its heads' weights away whole
        alive = np.isfinite(lse[s]).sum()
        assert abs(sums[s][0].sum() - alive) < 1e-9 * max(alive, 1)


def test_slots_in_any_order_and_their_rows_of_weights():
    rng = np.random.default_rng(50)
    lens = [70, 300, 20, 128]
    c, keys, _ = filled(rng, lens, 2, 128, 16)
    R, order = 3, [3, 1]
    q, q64 = bf16(rng, 2 * R, 4, 128)
    q64 = q64.reshape(2, R, 4, 128)
    weights = torch.ones(4, c.table.shape[1] * 16, device="cuda")
    lse = np.stack([O.attend(q64[i], keys[s], keys[s], 0.1, R)[1] for i, s in enumerate(order)])
    sph.kv_weigh(c, 0, q, torch.from_numpy(lse.reshape(2 * R, 4).astype(np.float32)).cuda(), R, 0.1, weights, slots=ints(order))
    for i, s in enumerate(order):
        within(host(weights)[s, :lens[s]], np.ones(lens[s]), *B.weigh(q64[i], keys[s], lse[i], 0.1, R), 128, R * 4)
    assert (host(weights)[[0, 2]] == 1).all()
    # slots that are none hold nothing
    sph.kv_weigh(c, 0, q, torch.zeros(2 * R, 4, device="cuda"), R, 0.1, weights, slots=ints([-1, 77]))
    assert (host(weights)[[0, 2]] == 1).all()


def test_attention_then_weights():
    # with the attention call's own log-sum-exp; a step's layers add up
    rng = np.random.default_rng(51)
    lens, R, heads, d = [900, 40, 333], 4, 4, 64
    c, keys, _ = filled(rng, lens, heads, d, 32)
    q, q64 = bf16(rng, 3 * R, 2 * heads, d)
    _, lse = sph.kv_attend(c, 0, q, R, 0.125, want_lse=True)
    weights = torch.full((3, c.table.shape[1] * 32), 5.0, device="cuda")
    sph.kv_weigh(c, 0, q, lse, R, 0.125, weights, fresh=True)
    sph.kv_weigh(c, 0, q, lse, R, 0.125, weights)
    for s in range(3):
        total, slack = B.weigh(q64.reshape(3, R, -1, d)[s], keys[s], host(lse).reshape(3, R, -1)[s], 0.125, R)
        before = np.full(lens[s], 5.0)
        before[-R:] = 0
        within(host(weights)[s, :lens[s]], before, 2 * total, 2 * slack, d, 4 * R * heads)


def test_masked_places_hold_anything():
    # a token whose key is no number says so at its own place only, and not at all where no row sees it; a row
    # without a log-sum-exp adds nothing, not even beside such a token
    rng = np.random.default_rng(52)
    n, R, d = 100, 4, 64
    c, keys, _ = filled(rng, [n], 1, d, 16)
    k = torch.zeros(1, 1, d, dtype=torch.bfloat16, device="cuda")
    k[0, 0, 5] = float("nan")
    full = c.lens.clone()
    c.lens.fill_(51)
    sph.kv_append(c, 0, k, k, 1)  # token 50
    c.lens.copy_(full)
    q, q64 = bf16(rng, R, 2, d)
    lse = torch.zeros(R, 2, device="cuda")
    weights = torch.zeros(1, c.table.shape[1] * 16, device="cuda")
    sph.kv_weigh(c, 0, q, lse, R, 0.125, weights)
    got = host(weights)[0]
    assert np.isnan(got[50]) and np.isfinite(np.delete(got, 50)).all()
    weights.zero_()
    sph.kv_weigh(c, 0, q, lse, R, 0.125, weights, window=40)
    assert np.isfinite(host(weights)).all() and (host(weights)[0, :57] == 0).all()
    weights.zero_()
    lse[1:] = -float("inf")
    lse[0] = -float("inf")
    sph.kv_weigh(c, 0, q, lse, R, 0.125, weights)
    assert (host(weights) == 0).all()
    # pages that are none
    c.table[0, 1] = -1
    lse.zero_()
    weights.fill_(2.0)
    sph.kv_weigh(c, 0, q, lse, R, 0.125, weights)
    assert (host(weights)[0, 16:32] == 2).all() and (host(weights)[0, :16] > 2).all()


def test_captured_replayed_and_again_the_same():
    rng = np.random.default_rng(53)
    lens = [1500, 900, 2000]
    c, keys, _ = filled(rng, lens, 2, 128, 16)
    R = 5
    q, q64 = bf16(rng, 3 * R, 8, 128)
    weights = torch.zeros(3, c.table.shape[1] * 16, device="cuda")
    lse = torch.zeros(3 * R, 8, device="cuda")
    ws = torch.empty(max(1, sph.kv_weigh_workspace(c, 8, 3, R)), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        sph.kv_weigh(c, 0, q, lse, R, 0.05, weights, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sph.kv_weigh(c, 0, q, lse, R, 0.05, weights, workspace=ws)
    for turn in range(4):
        q.copy_(bf16(rng, 3 * R, 8, 128)[0])
        lse.copy_(sph.kv_attend(c, 0, q, R, 0.05, want_lse=True)[1])
        eager = torch.zeros_like(weights)
        sph.kv_weigh(c, 0, q, lse, R, 0.05, eager)
        weights.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(weights, eager)
        assert abs(float(weights.sum()) / (3 * R * 8) - 1) < 1e-5
