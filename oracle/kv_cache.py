"""Oracle of the paged 4-bit key/value cache: plain NumPy in 64 bits, from the
definitions, on logical tokens and lists of pages.  It knows nothing of how a
page orders its bytes.

Format: 32 values share 2^e and are each one of the E2M1 values (OCP
microscaling FP4, which leaves the choice of e open).  Here e = floor(log2 m) - 2
with m the largest magnitude rounded to two significant bits, ties to even, and e in [-127, 125].
"""

from __future__ import annotations

import numpy as np

GROUP = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """The values that the cache holds for x [..., D] (finite, D a multiple of 32),
    as float64."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    top = np.abs(g).max(-1)
    out = np.zeros_like(g)
    for at in np.argwhere(top > 0):
        at = tuple(at)
        # the least e for which the largest element rounds to at most 6
        f, b = np.frexp(top[at])                   # top = f 2^b, f in [0.5, 1)
        e = b - 3                                  # 2^(b-1) <= top: e = floor(log2 top) - 2
        if f >= 0.875:                             # 7/8: two significant bits round up to 2^b
            e += 1
        e = int(min(max(e, -127), 125))            # 6 * 2^126 is no bf16
        out[at] = np.sign(g[at]) * nearest_e2m1(np.abs(g[at]) / 2.0 ** e) * 2.0 ** e
    return out.reshape(x.shape)


def nearest_e2m1(a):
    """Nearest E2M1 magnitude, ties to the code with an even last bit, saturating."""
    a = np.asarray(a, dtype=np.float64)
    d = np.abs(a[..., None] - E2M1)
    lo = d.argmin(-1)                              # the lower of two equally near
    hi = np.minimum(lo + 1, 7)
    tie = d[..., 0] * 0 + np.take_along_axis(d, lo[..., None], -1)[..., 0] == \
        np.take_along_axis(d, hi[..., None], -1)[..., 0]
    code = np.where(tie & (hi > lo) & (lo % 2 == 1), hi, lo)
    return E2M1[code]


def attend(q, k, v, scale, rows, window=0):
    """One session: q [R, Hq, D] (its first `rows` count), k, v [n, Hkv, D] as the
    cache holds them.  Returns out, lse, the weighted sum of |v| (what bounds the
    rounding of the weights) and the largest scale * sum |q k| of each row."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    R, Hq, D = q.shape
    n, Hkv, _ = k.shape
    G = Hq // Hkv
    out = np.zeros((R, Hq, D))
    mag = np.zeros((R, Hq, D))
    lse = np.full((R, Hq), -np.inf)
    size = np.zeros((R, Hq))
    for r in range(min(rows, R)):
        p = n - rows + r
        first = max(0, p - window + 1) if window else 0
        if p < first:
            continue
        kk, vv = k[first:p + 1], v[first:p + 1]
        for h in range(Hq):
            x = scale * kk[:, h // G] @ q[r, h]
            top = x.max()
            w = np.exp(x - top)
            z = w.sum()
            out[r, h] = w @ vv[:, h // G] / z
            mag[r, h] = w @ np.abs(vv[:, h // G]) / z
            lse[r, h] = top + np.log(z)
            size[r, h] = scale * (np.abs(kk[:, h // G]) @ np.abs(q[r, h])).max()
    return out, lse, mag, size


class Pages:
    """Tables, lengths and counts of a pool, with what each call does to them; the
    contents of pages are tracked as `content[page]`, any value."""

    def __init__(self, n_pages, n_slots, max_pages, page):
        self.page = page
        self.table = np.full((n_slots, max_pages), -1, np.int64)
        self.lens = np.zeros(n_slots, np.int64)
        self.refs = np.zeros(n_pages, np.int64)
        self.content = list(range(n_pages))

    def _held(self, n):
        return -(-int(n) // self.page)

    def grow(self, add):
        add = np.maximum(add, 0)
        before = self.refs.copy()
        free = [int(p) for p in np.flatnonzero(before <= 0)]
        wants, short = [], 0
        for s, (n, more) in enumerate(zip(self.lens, add)):
            have, want = self._held(n), self._held(n + more)
            if want > self.table.shape[1]:
                short += 1
                continue
            if more > 0 and n % self.page and before[self.table[s, n // self.page]] > 1:
                wants.append((s, n // self.page, True))
            wants += [(s, c, False) for c in range(have, want)]
        lacking = max(0, len(wants) - len(free))
        if short == 0 and lacking == 0:
            for (s, c, copy), p in zip(wants, free):
                if copy:
                    old = self.table[s, c]
                    self.refs[old] -= 1
                    self.content[p] = self.content[old]
                self.table[s, c] = p
                self.refs[p] = 1
            self.lens += add
        return lacking, short

    def trim(self, kept):
        for s in range(len(self.lens)):
            keep = max(int(kept[s]), 0)
            if keep < self.lens[s]:
                for c in range(self._held(keep), self._held(self.lens[s])):
                    self.refs[self.table[s, c]] -= 1
                    self.table[s, c] = -1
                self.lens[s] = keep

    def fork(self, parents, children):
        self.trim([0 if s in set(children) else n for s, n in enumerate(self.lens)])
        for p, c in zip(parents, children):
            self.table[c] = self.table[p]
            self.lens[c] = self.lens[p]
            for page in self.table[p, :self._held(self.lens[p])]:
                self.refs[page] += 1

    def compact(self):
        live = [int(p) for p in np.flatnonzero(self.refs > 0)]
        holes = [p for p in range(len(live)) if self.refs[p] <= 0]
        movers = [p for p in live if p >= len(live)]
        to = dict(zip(movers, holes))
        for a, b in to.items():
            self.content[b] = self.content[a]
            self.refs[b] = self.refs[a]
            self.refs[a] = 0
        self.refs[len(live):] = 0
        self.table = np.array([[to.get(int(p), int(p)) for p in row] for row in self.table])
        return len(live)
