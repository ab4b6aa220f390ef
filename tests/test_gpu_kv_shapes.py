"""Every instance of the cache attention at sizes where its rings turn many times:
each head size, row tiles and waves, with one share of the tokens, a few and many,
one workgroup for a head's rows and several, with and without a window. Against
64-bit products on the GPU of what the cache holds (kv_read, checked elsewhere),
within the bounds derived in test_gpu_kv.py."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph

import kv_rules
from kv_build import cache_of
from test_gpu_kv import say

pytestmark = pytest.mark.gpu

# q heads, kv heads, d, sessions, rows, longest, window; then the shape meant: row
# tiles, waves that share rows, join kind
SHAPES = [
    (2, 1, 64, 1, 1, 100, 50, (1, 4, 0)), (2, 1, 64, 1, 9, 100, 0, (1, 4, 0)), (4, 1, 64, 1, 200, 1500, 0, (1, 4, 1)),
    (1, 1, 64, 1, 1, 1500, 0, (1, 4, 2)), (16, 2, 64, 64, 33, 100, 50, (2, 2, 0)), (21, 3, 64, 16, 100, 100, 0, (2, 2, 0)),
    (32, 8, 64, 64, 5, 3000, 0, (1, 4, 0)), (14, 2, 64, 40, 33, 100, 50, (2, 4, 0)), (14, 2, 64, 1, 300, 3000, 0, (2, 4, 1)),
    (14, 2, 64, 1, 100, 12000, 0, (2, 4, 2)), (8, 8, 64, 64, 33, 1500, 0, (4, 4, 0)), (10, 2, 64, 5, 500, 1500, 0, (4, 4, 0)),
    (3, 1, 64, 40, 33, 6000, 0, (4, 4, 1)), (4, 2, 64, 3, 200, 12000, 0, (4, 4, 2)),
    (1, 1, 128, 1, 1, 100, 50, (1, 4, 0)), (2, 1, 128, 1, 9, 100, 50, (1, 4, 0)), (5, 1, 128, 1, 100, 1500, 0, (1, 8, 0)),
    (1, 1, 128, 1, 1, 1500, 0, (1, 4, 2)), (40, 8, 128, 64, 7, 100, 50, (2, 2, 0)), (16, 2, 128, 16, 100, 100, 0, (2, 2, 0)),
    (40, 8, 128, 64, 5, 100, 50, (2, 4, 0)), (14, 2, 128, 16, 64, 100, 700, (2, 4, 0)), (5, 1, 128, 1, 500, 3000, 0, (1, 8, 0)),
    (8, 1, 128, 1, 100, 12000, 0, (1, 8, 2)), (8, 8, 128, 64, 33, 700, 700, (4, 4, 0)), (56, 8, 128, 1, 500, 700, 0, (4, 4, 0)),
    (14, 2, 128, 2, 300, 3000, 0, (1, 8, 0)), (1, 1, 128, 40, 33, 12000, 0, (4, 4, 2)),
    (56, 8, 256, 40, 3, 100, 50, (1, 2, 0)), (21, 3, 256, 5, 100, 100, 0, (1, 2, 0)), (8, 1, 256, 2, 200, 12000, 0, (2, 8, 1)),
    (3, 1, 256, 1, 1, 100, 50, (1, 4, 0)), (4, 1, 256, 1, 5, 100, 0, (1, 4, 0)), (1, 1, 256, 1, 1, 700, 0, (1, 4, 1)),
    (1, 1, 256, 1, 1, 1500, 0, (1, 4, 2)),
    (9, 3, 128, 16, 2, 3000, 0, (1, 4, 1)), (4, 2, 128, 1, 100, 3000, 0, (1, 8, 1)), (21, 3, 128, 2, 100, 3000, 0, (2, 4, 1)),
    (2, 2, 128, 2, 100, 16001, 0, (2, 4, 2)), (112, 16, 128, 1, 33, 16001, 0, (4, 4, 1)), (6, 2, 256, 1, 33, 700, 0, (2, 8, 0)),
    (2, 2, 256, 2, 33, 16001, 0, (2, 8, 2)),
    # started by their lengths
    (24, 8, 64, 64, 5, 3000, 0, (1, 4, 0)), (8, 8, 64, 64, 33, 3000, 0, (2, 4, 0)), (80, 16, 64, 64, 8, 3000, 0, (4, 4, 0)),
    (6, 2, 128, 256, 1, 3000, 0, (1, 8, 0)), (24, 8, 128, 64, 8, 3000, 0, (2, 4, 0)), (40, 8, 128, 64, 8, 3000, 0, (4, 4, 0)),
    (8, 8, 256, 64, 9, 3000, 0, (1, 4, 0)), (9, 3, 256, 256, 8, 3000, 0, (2, 8, 0)),
]


def shape_of(case):
    hq, hkv, d, n, R, most, window, _ = case
    mt, wt, _, splits, _ = kv_rules.attend_shape(d, n, R, hkv, hq, most, window)
    return mt, wt, kv_rules.join_kind(splits)


@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join(map(str, c[:7])))
def test_shape(case):
    hq, hkv, d, n, R, most, window, want = case
    assert shape_of(case) == want
    say("shape", case)
    rng = np.random.default_rng(hq * 7 + d + R + most)
    lens = [most] + [int(x) for x in rng.integers(0, most + 1, n - 1)]
    rows = [R] + [int(x) for x in rng.integers(0, R + 1, n - 1)]
    page = int(rng.choice([16, 32, 64, 128]))
    c = cache_of(rng, lens, hkv, d, page)
    g = torch.Generator(device="cuda")
    g.manual_seed(most + R)
    full = torch.tensor(lens, dtype=torch.int32).cuda()
    for name in ("k", "v"):
        x = torch.randn(n * most, hkv, d, generator=g, device="cuda").to(torch.bfloat16)
        k = x if name == "k" else k
    sph.kv_append(c, 0, k, x, most, rows=full)
    k, v = (t.view(n, most, hkv, d) for t in sph.kv_read(c, 0, most, rows=full))
    q = (1.5 * torch.randn(n * R, hq, d, generator=g, device="cuda")).to(torch.bfloat16)
    scale = d ** -0.5
    out, lse = sph.kv_attend(c, 0, q, R, scale, rows=torch.tensor(rows, dtype=torch.int32).cuda(), window=window,
                             max_len=most, want_lse=True)
    assert bool(torch.isfinite(out).all())
    out, lse, q = out.view(n, R, hq, d).double(), lse.view(n, R, hq).double(), q.view(n, R, hq, d)
    worst = 0.0
    for s in range(n):
        L, r = lens[s], rows[s]
        assert not out[s, r:].any() and bool(torch.isneginf(lse[s, r:]).all())
        if L == 0 or r == 0:
            assert not out[s].any() and bool(torch.isneginf(lse[s]).all())
            continue
        pos = torch.arange(L - r, L, device="cuda")
        j = torch.arange(L, device="cuda")
        see = (j[None] <= pos[:, None]) & ((j[None] > pos[:, None] - window) if window else True)
        for h in range(hkv):
            G = hq // hkv
            qq = q[s, :r, h * G:(h + 1) * G].double().reshape(-1, d)
            kk, vv = k[s, :L, h].double(), v[s, :L, h].double()
            mask = see.repeat_interleave(G, 0)
            x = (scale * qq @ kk.T.contiguous()).masked_fill(~mask, -np.inf)
            size = (scale * qq.abs() @ kk.abs().T.contiguous()).masked_fill(~mask, 0).amax(-1)
            none = ~mask.any(-1)
            top = x.amax(-1, keepdim=True).clamp(min=-1e300)
            p = (x - top).exp()
            z = p.sum(-1, keepdim=True)
            p = p / z.clamp(min=1e-300)
            o, mag = p @ vv, p @ vv.abs()
            e = (d + 8) * 2.0 ** -24 * size
            got = out[s, :r, h * G:(h + 1) * G].reshape(-1, d)
            bound = 2.0 ** -8 * o.abs() + (2.0 ** -8 + 2.0 ** -18 + 4 * e[:, None]) * mag + 1e-37
            worst = max(worst, float(((got - o).abs() / bound).max()))
            ref = (top + z.log()).squeeze(-1)
            gl = lse[s, :r, h * G:(h + 1) * G].reshape(-1)
            assert torch.equal(torch.isneginf(gl), none)
            off = (gl - ref).abs()[~none] - (2 * e + 2.0 ** -20 * ref.abs().clamp(min=1) + L * 2.0 ** -24)[~none]
            assert bool((off <= 0).all())
    say("worst output error: %.3f of its bound" % worst)
    assert worst <= 1.0


@pytest.mark.parametrize("hkv,d,n", [(8, 128, 40), (4, 64, 255), (2, 256, 256), (300, 64, 2)])
def test_order_of_sessions(hkv, d, n):
    # sessions are started by their lengths: what each answers does not depend on it
    say("order", hkv, d, n)
    rng = np.random.default_rng(hkv + n)
    most = 2600
    lens = [int(x) for x in rng.integers(0, most + 1, n)]
    lens[:n // 3] = [most] * (n // 3)                 # ties, and sessions of nothing
    lens[n // 2] = 0
    c = cache_of(rng, lens, hkv, d, 64)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    c.pool.random_(0, 128, generator=g)               # any codes, scales of 2^-127 ... 2^0
    q = torch.randn(n, hkv, d, generator=g, device="cuda").to(torch.bfloat16)
    want, wl = sph.kv_attend(c, 0, q, 1, 0.1, max_len=most, want_lse=True)
    assert bool(torch.isfinite(want).all()) and bool(torch.isneginf(wl[n // 2]).all())
    at = torch.from_numpy(rng.permutation(n).astype(np.int32)).cuda()
    out, lse = sph.kv_attend(c, 0, q[at.long()], 1, 0.1, slots=at, max_len=most, want_lse=True)
    assert torch.equal(out, want[at.long()]) and torch.equal(lse, wl[at.long()])
    one = int(np.argmax(lens)), int(np.argmin(lens))
    for s in one:                                     # alone: the same but for the order of sums
        slot = torch.tensor([s], dtype=torch.int32).cuda()
        o, l = sph.kv_attend(c, 0, q[s:s + 1], 1, 0.1, slots=slot, max_len=most, want_lse=True)
        # the weights and each output round to bf16
        v = want[s].float().abs().max()
        assert float((o.float() - want[s:s + 1].float()).abs().max()) <= float(v) * 2.0 ** -5
        assert torch.allclose(l, wl[s:s + 1], rtol=2.0 ** -18, atol=2.0 ** -12)
