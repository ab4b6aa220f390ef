"""Caches for the GPU tests: random keys and values appended through the library
into pages in random order, and the same as the oracle holds them."""

import numpy as np
import torch

import paper_2607_13093_amd as sph
from oracle import kv_cache as O


def bf16(rng, *shape, scale=1.0):
    """Random normals as bf16 on the GPU, and the same in float64."""
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)
    return t.cuda(), t.to(torch.float64).numpy()


def tables(rng, lens, page, n_slots=None, n_pages=None, extra=1):
    """Pages of the slots in random order, as (table, refs) numpy."""
    n_slots = len(lens) if n_slots is None else n_slots
    counts = [-(-n // page) for n in lens]
    n_pages = sum(counts) + 3 if n_pages is None else n_pages
    table = np.full((n_slots, max(counts + [1]) + extra), -1, np.int32)
    order = rng.permutation(n_pages)[:sum(counts)]
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = order[at:at + c]
        at += c
    refs = np.zeros(n_pages, np.int32)
    refs[order] = 1
    return table, refs


def cache_of(rng, lens, heads, d, page, layers=1, fill=0xFF, **kw):
    """An unwritten cache: every byte is `fill` (0xFF: NaN scales)."""
    table, refs = tables(rng, lens, page, **kw)
    pool = torch.full((layers, len(refs), sph.kv_page_bytes(heads, d, page)), fill, dtype=torch.uint8, device="cuda")
    full = np.zeros(len(table), np.int32)
    full[:len(lens)] = lens
    return sph.KvCache(pool, torch.from_numpy(table).cuda(), torch.from_numpy(full).cuda(),
                       torch.from_numpy(refs).cuda(), heads, d, page)


def filled(rng, lens, heads, d, page, layer=0, layers=1, **kw):
    """(cache, keys, values): the latter lists of float64 [len, heads, d] per session, as held."""
    c = cache_of(rng, lens, heads, d, page, layers=layers, **kw)
    n, R = len(lens), max(max(lens), 1)
    k, k64 = bf16(rng, n * R, heads, d)
    v, v64 = bf16(rng, n * R, heads, d)
    rows = torch.tensor(lens, dtype=torch.int32).cuda()
    sph.kv_append(c, layer, k, v, R, rows=rows)
    hold = [[O.quantize(x.reshape(n, R, heads, d)[s, :lens[s]]) for s in range(n)] for x in (k64, v64)]
    return c, hold[0], hold[1]


def host(t):
    return t.detach().to("cpu").to(torch.float64 if t.is_floating_point() else t.dtype).numpy()
