"""Oracle of eviction from the paged cache and of the weights that it goes by: plain
NumPy in 64 bits, from the definitions, one slot and one row at a time."""

from __future__ import annotations

import math

import numpy as np


def choose(weights, n, keep, front, recent):
    """Positions that a slot of n tokens keeps: the first `front`, the last `recent`,
    and of the others those with the largest weights, a NaN the smallest, equal ones by
    position, `keep` in all if that is more."""
    front = min(front, n)
    back = max(front, n - min(recent, n))
    must = list(range(front)) + list(range(back, n))

    def order(j):
        w = float(weights[j])
        return (1, 0.0, j) if math.isnan(w) else (0, -w, j)

    others = sorted(range(front, back), key=order)
    return sorted(must + others[:max(0, min(keep, n) - len(must))])


def evict(table, lens, refs, weights, keep, first, recent, page):
    """All slots: (kept positions, table, lens, refs), the inputs unchanged."""
    table, lens, refs = table.copy(), lens.copy(), refs.copy()
    before = refs.copy()
    kept = []
    for s in range(len(lens)):
        n = int(lens[s])
        held = -(-n // page)
        last = max([c + 1 for c in range(held) if table[s, c] >= 0 and before[table[s, c]] > 1], default=0)
        kept.append(choose(weights[s], n, int(keep[s]), max(int(first), last * page), int(recent)))
        for c in range(-(-len(kept[-1]) // page), held):
            if table[s, c] >= 0:
                refs[table[s, c]] -= 1
            table[s, c] = -1
        lens[s] = len(kept[-1])
    return kept, table, lens, refs


def weigh(q, k, lse, scale, rows, window=0):
    """One session: what each of its n tokens receives from its rows. q [R, Hq, D] (the
    first `rows` count), k [n, Hkv, D] as the cache holds them, lse [R, Hq]. Returns the
    sums [n], and what bounds their rounding: the sums weighted by 1 + the size of the
    score and of the log-sum-exp."""
    q, k, lse = (np.asarray(a, dtype=np.float64) for a in (q, k, lse))
    n, hkv, _ = k.shape
    group = q.shape[1] // hkv
    total, slack = np.zeros(n), np.zeros(n)
    for r in range(min(rows, q.shape[0])):
        p = n - rows + r
        first = max(0, p - window + 1) if window else 0
        if p < first:
            continue
        for h in range(q.shape[1]):
            x = scale * k[first:p + 1, h // group] @ q[r, h]
            size = scale * np.abs(k[first:p + 1, h // group]) @ np.abs(q[r, h])
            if lse[r, h] == -np.inf:
                continue
            w = np.exp(x - lse[r, h])
            total[first:p + 1] += w
            slack[first:p + 1] += w * (1 + size + abs(lse[r, h]))
    return total, slack
