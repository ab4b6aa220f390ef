"""Shared attention, token weights and eviction together, as a server's steps use them:
prompts are branched, branches decode windows, tokens' weights add up over the layers,
and sessions over their budget drop tokens, while the 64-bit oracle follows what each
slot holds."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph
from oracle import kv_budget as B
from oracle import kv_cache as O

from kv_build import bf16, host

pytestmark = pytest.mark.gpu


def say(*a):
    print("[gpu]", *a, flush=True)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


@pytest.mark.parametrize("heads,group,d,page", [(2, 4, 64, 16), (1, 2, 128, 32), (2, 2, 256, 16)])
def test_steps_of_branches_at_a_budget(heads, group, d, page):
    rng = np.random.default_rng(d)
    layers, slots, R, prompt, budget = 2, 5, 3, 130, 170
    Hq, scale = heads * group, d ** -0.5
    c = sph.KvCache.empty(layers, 120, slots, 40, heads, d, page)
    c.pool.fill_(0xFF)
    width = 40 * page
    weights = torch.full((slots, width), float("nan"), device="cuda")  # what a slot's former session left
    k = [[np.zeros((0, heads, d)) for _ in range(slots)] for _ in range(layers)]
    v = [[np.zeros((0, heads, d)) for _ in range(slots)] for _ in range(layers)]

    def step(rows, most):
        """One window of every slot: all layers' attention and weights, checked."""
        assert host(sph.pages_grow(c, ints(rows))).tolist() == [0, 0]
        plan = sph.kv_share(c, Hq, most, rows=ints(rows), n_sessions=slots)
        for layer in range(layers):
            kt, k64 = bf16(rng, slots * most, heads, d)
            vt, v64 = bf16(rng, slots * most, heads, d)
            q, q64 = bf16(rng, slots * most, Hq, d)
            sph.kv_append(c, layer, kt, vt, most, rows=ints(rows))
            for s in range(slots):
                for held, x in ((k, k64), (v, v64)):
                    held[layer][s] = np.concatenate([held[layer][s], O.quantize(x.reshape(slots, most, heads, d)[s, :rows[s]])])
            before = host(weights).copy()
            out, lse = sph.kv_attend_shared(c, layer, q, plan, scale, want_lse=True)
            sph.kv_weigh(c, layer, q, lse, most, scale, weights, rows=ints(rows), fresh=layer == 0)
            o, after = host(out).reshape(slots, most, Hq, d), host(weights)
            l = host(lse).reshape(slots, most, Hq)
            for s in range(slots):
                q_s, n = q64.reshape(slots, most, Hq, d)[s], len(k[layer][s])
                want, wl, mag, size = O.attend(q_s, k[layer][s], v[layer][s], scale, rows[s])
                err = (d + 8) * 2.0 ** -24 * size
                tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -18 + 4 * err[..., None]) * mag + 1e-30
                assert (np.abs(o[s] - want) <= tol).all(), (layer, s)
                total, slack = B.weigh(q_s, k[layer][s], l[s], scale, rows[s])
                was = before[s, :n].copy()
                if layer == 0:
                    was[n - rows[s]:] = 0
                tol = 2.0 ** -24 * (d + 12) * slack + (2.0 ** -20 + most * Hq * 2.0 ** -24) * total + 2.0 ** -24 * np.abs(was + total)
                assert (np.abs(after[s, :n] - was - total) <= tol).all(), (layer, s)

    def evict(keep, first, recent):
        was = {n: host(t).copy() for n, t in (("table", c.table), ("lens", c.lens), ("refs", c.refs))}
        w = host(weights).astype(np.float32)
        _, kept = sph.pages_evict(c, weights, ints(keep), first, recent, want_kept=True)
        want, table, lens, refs = B.evict(was["table"], was["lens"], was["refs"], w, keep, first, recent, page)
        np.testing.assert_array_equal(host(c.table), table)
        np.testing.assert_array_equal(host(c.lens), lens)
        np.testing.assert_array_equal(host(c.refs), refs)
        for s in range(slots):
            np.testing.assert_array_equal(host(kept)[s, :len(want[s])], want[s])
            for layer in range(layers):
                k[layer][s], v[layer][s] = k[layer][s][want[s]], v[layer][s][want[s]]
        return lens

    step([prompt, 0, 0, 0, 60], prompt)
    sph.pages_fork(c, ints([0, 0]), ints([1, 3]))
    for s in (1, 3):
        weights[s] = weights[0]
        for layer in range(layers):
            k[layer][s], v[layer][s] = k[layer][0], v[layer][0]
    say("branched", heads, group, d, page)
    for turn in range(3):
        step([R, 1, 0, R - 1, R], R)
        step([40, 35, 0, 50, 60], 60)
        lens = evict([budget] * slots, 4, 2 * R)
        say("turn", turn, "held", lens.tolist())
    # the prompt's whole pages are still the branches' own
    shared = prompt // page
    table = host(c.table)
    assert (table[0, :shared] == table[1, :shared]).all() and (table[0, :shared] == table[3, :shared]).all()
    assert (host(c.refs)[table[0, :shared]] == 3).all()
    # a branch that ends frees only what was its own
    sph.pages_trim(c, ints([1 << 20, 0, 1 << 20, 1 << 20, 1 << 20]))
    k[0][1], k[1][1], v[0][1], v[1][1] = (x[:0] for x in (k[0][1], k[1][1], v[0][1], v[1][1]))
    assert (host(c.refs)[table[0, :shared]] == 2).all()
    step([R, 0, 2, R, 1], R)
