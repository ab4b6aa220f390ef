"""Performance cases of the paged 4-bit key/value cache.

A speculative step of a server: the cache grows by each session's window of rows, the window's keys and values
are appended, its queries attend over the cache, and after verification the pages of rejected drafts are given
back. Prompts run through the same calls with many rows, answers are branched by forking sessions, and a pool
with holes is compacted.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare`` makes a case's inputs,
``run`` is one pass (the plain form in elementary torch operations, or the library's calls where ``own`` is
true), ``work`` and ``exact`` say what a pass has to do and what 64-bit arithmetic gives.

Paths
  attend  queries of every session's last rows over its cache: outputs and log-sum-exp
  append  keys and values quantised into their pages, and read back as the values they stand for
  step    rejected rows given back, pages for the window, append and attend, on one layer
  turn    the pages of a step alone: trim, then grow, tables and reference counts
  fork    sessions branched from others, then grown (shared last pages are copied, in every layer)
  compact live pages moved to the front of the pool, in every layer

Ranges: 1 to 256 sessions with windows of 1 to 9 rows or prompts of up to some thousand, caches of one token
to 65536, 1 to 64 query heads on 1 to 16 key/value heads, head sizes 64, 128 and 256, pages of 16 to 128
tokens, with and without a sliding window. Hidden sizes 512, 4096, 5120 and 8192 are 4 to 64 heads of 128.
"""

import math

import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, path, **kw):
    c = {"name": name, "path": path, "sessions": 1, "rows": 5, "ragged_rows": False, "len_lo": 1, "len_hi": 4096,
         "q_heads": 32, "kv_heads": 8, "d": 128, "page": 64, "window": 0, "layers": 1, "children": 0, "pages": 0}
    c.update(kw)
    return c


def listed():
    return [
        # one user's plain decoding of a short text: a few microseconds, launches and host code count
        _case("attend_one_short", "attend", rows=1, len_lo=300, len_hi=300, page=16),
        # one user's window of four drafts over a long document: few rows, one long axis
        _case("attend_window_long", "attend", len_lo=65521, len_hi=65521),
        # 64 users' windows of very different lengths, small pages
        _case("attend_batched", "attend", sessions=64, len_hi=8192, page=16),
        # a large server batch: 256 sessions, 64 query heads, the cache is a stream from memory
        _case("attend_dense", "attend", sessions=256, rows=8, len_hi=16384, q_heads=64),
        # a chunk of a long prompt behind what the cache holds already: matrix products
        _case("attend_prompt_chunk", "attend", rows=4099, len_lo=16001, len_hi=16001, q_heads=40),
        # several prompts of different lengths with a sliding window and a small head
        _case("attend_prompt_sliding", "attend", sessions=4, rows=2047, ragged_rows=True, len_lo=2047, len_hi=5000,
              q_heads=16, kv_heads=16, d=64, page=32, window=1024),
        # the appended window of a batch of users, read back: launches count
        _case("append_window", "append", sessions=64, len_lo=5, len_hi=8192, page=16),
        # prompts written into the cache and handed on as values
        _case("append_prompt", "append", sessions=8, rows=4096, ragged_rows=True, len_lo=4096, len_hi=6000),
        # one layer of a step: 128 users, large heads
        _case("step_batch", "step", sessions=128, len_lo=5, len_hi=4096, q_heads=16, kv_heads=4, d=256, page=32),
        # the pages of a large batch's step: windows of eight rows rejected and grown again
        _case("turn_dense", "turn", sessions=256, rows=8, len_lo=8, len_hi=16384, kv_heads=1, d=64,
              pages=65536),
        # eight prompts branched into 31 answers each, 32 layers: shared last pages are copied
        _case("fork_answers", "fork", sessions=8, children=248, len_lo=40, len_hi=4096, layers=32),
        # half of a pool of 16 layers has holes: it is moved to the front
        _case("compact_pool", "compact", sessions=64, len_lo=1, len_hi=4096, layers=16, pages=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        path = rng.choice(["attend", "attend", "attend", "prompt", "append", "step", "turn", "fork", "compact"])
        d = rng.choice([64, 128, 128, 128, 256])
        kv = rng.choice([1, 2, 4, 8, 8, 16])
        group = rng.choice([1, 2, 3, 4, 5, 7, 8])
        c = _case("", path, d=d, kv_heads=kv, q_heads=kv * group, page=rng.choice([16, 32, 64, 128]),
                  sessions=_log(rng, 1, 256), rows=rng.choice([1, 1, 2, 3, 5, 6, 7, 8, 9]),
                  len_hi=_log(rng, 1, 65536), window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]))
        c["len_lo"] = rng.choice([1, c["len_hi"]])
        if path == "prompt" or path == "append" and rng.random() < 0.5:
            c["rows"] = _log(rng, 10, 4099)
            c["sessions"] = _log(rng, 1, 16)
            c["len_hi"] = c["rows"] + rng.choice([0, _log(rng, 1, 12000)])
            c["len_lo"] = c["rows"]
            c["ragged_rows"] = rng.random() < 0.5
        if path == "prompt":
            c["path"] = "attend"
        if path in ("append", "step", "turn"):
            c["len_hi"] = max(c["len_hi"], c["rows"])
            c["len_lo"] = max(c["len_lo"], c["rows"])
        if path in ("turn", "fork", "compact"):
            c["window"] = 0
        if path == "turn":
            c["pages"] = _log(rng, 1024, 65536)
        if path in ("fork", "compact"):
            c["layers"] = _log(rng, 1, 32)
            c["len_hi"] = min(c["len_hi"], 4096)
            c["len_lo"] = min(c["len_lo"], c["len_hi"])
        if path == "fork":
            c["sessions"] = _log(rng, 1, 16)
            c["children"] = c["sessions"] * rng.choice([1, 2, 3, 7, 15])
        if path == "compact":
            c["pages"] = _log(rng, 256, 4096)
        if _fits(c):
            return c


def _fits(c):
    """No more than the largest listed cases, in the cache, in the scores and in the products."""
    tokens = (c["sessions"] + c["children"]) * c["len_hi"]
    pages = (c["sessions"] + c["children"]) * -(-c["len_hi"] // c["page"])
    page_bytes = c["kv_heads"] * c["page"] * c["d"] * 17 // 16
    pool = c["layers"] * max(pages, c["pages"]) * page_bytes
    pairs = c["sessions"] * c["q_heads"] * c["rows"] * c["len_hi"]
    if c["path"] in ("turn", "fork", "compact"):
        return pool <= 4 << 30 and (c["path"] != "compact" or pages <= 0.6 * c["pages"]) and (
            c["path"] != "turn" or pages <= c["pages"])
    return tokens * c["kv_heads"] * c["d"] <= 256 * 16384 * 8 * 128 and pairs <= 40 * 4099 * 16001 and (
        pairs * c["d"] <= 40 * 4099 * 16001 * 128)


# ---------------------------------------------------------------------------
# sizes that a case's seedless part fixes
# ---------------------------------------------------------------------------

def _lens(case):
    """Lengths (the window's rows among them) and window rows of every session, from the case alone."""
    n, lo, hi = case["sessions"], case["len_lo"], case["len_hi"]
    # a fixed spread between the bounds, both of them taken
    lens = [lo + (hi - lo) * ((i * 37) % n) // max(n - 1, 1) for i in range(n)] if n > 1 else [hi]
    rows = [case["rows"] - (i * case["rows"] // (2 * n) if case["ragged_rows"] else 0) for i in range(n)]
    return lens, rows


def _pages_of(n, page):
    return -(-n // page)


def _page_bytes(case):
    return case["kv_heads"] * case["page"] * case["d"] * 17 // 16


def _visible(case):
    """Pairs of a row and a position that it sees, over all sessions, and the positions that any row sees."""
    lens, rows = _lens(case)
    pairs = seen = 0
    for n, r in zip(lens, rows):
        w = case["window"] or n
        first, last = n - r, n - 1
        lo, hi = max(first, 0), min(last, w - 1)  # rows that see all before them
        pairs += (lo + hi + 2) * (hi - lo + 1) // 2 if hi >= lo else 0
        pairs += max(0, last - max(first, w, 0) + 1) * w
        seen += n - max(0, max(first, 0) - w + 1)
    return pairs, seen


def work(case):
    c = case
    lens, rows = _lens(c)
    path, vec = c["path"], c["kv_heads"] * c["d"]
    m = sum(rows)
    held = 2 * vec * 17 / 32  # bytes of one token's keys and values in the cache
    pairs, seen = _visible(c)
    attend = {"bytes": seen * held + m * c["q_heads"] * (4 * c["d"] + 4) + 4 * sum(_pages_of(n, c["page"]) for n in lens),
              "flops": 4 * pairs * c["q_heads"] * c["d"]}
    if path == "attend":
        return attend
    if path == "append":  # values in, codes out, codes in, values out
        return {"bytes": 2 * m * (4 * vec + held), "flops": 4 * m * vec}
    taken = [_pages_of(n, c["page"]) - _pages_of(n - r, c["page"]) for n, r in zip(lens, rows)]
    turn = {"bytes": 4 * max(c["pages"], sum(_pages_of(n, c["page"]) for n in lens)) + 32 * c["sessions"] + 16 * sum(taken),
            "flops": 0}
    if path == "turn":
        return turn
    if path == "step":
        return {"bytes": attend["bytes"] + m * (4 * vec + held) + turn["bytes"], "flops": attend["flops"]}
    if path == "fork":
        per = c["children"] // c["sessions"]
        copied = sum(per for n in lens if n % c["page"])
        return {"bytes": 2 * copied * c["layers"] * _page_bytes(c) + per * 12 * sum(_pages_of(n, c["page"]) for n in lens),
                "flops": 0}
    moved = _moved(c)
    return {"bytes": 2 * moved * c["layers"] * _page_bytes(c) + 8 * c["pages"] + 8 * sum(_pages_of(n, c["page"]) for n in lens),
            "flops": 0}


def _moved(case):
    """About how many pages a compaction moves: live pages lie anywhere in the pool."""
    live = sum(_pages_of(n, case["page"]) for n in _lens(case)[0])
    return live * (1 - live / case["pages"])


# ---------------------------------------------------------------------------
# the format: 32 values share a power of two, each is an E2M1 code
# ---------------------------------------------------------------------------

def _codes(x):
    """Codes (0 .. 15, sign in bit 3) and scale bytes of fp32 vectors x [..., D] in groups of 32."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    _, e = torch.frexp(top)                      # top = f 2^e, f in [0.5, 1)
    f = torch.ldexp(top, -e)
    e = e - 1 + (f >= 0.875).to(e.dtype) - 2     # from 1.75 on the top would round past 6
    e = torch.where(top > 0, e.clamp(-127, 127), -127)
    a = torch.ldexp(g.abs(), -e.unsqueeze(-1))
    _, b = torch.frexp(a.clamp(1.0, 6.0))        # 1 .. 3: the step is 0.5, 1 or 2
    step = torch.ldexp(torch.ones_like(a), b - 2)
    q = torch.round(a / step) * step             # ties to even
    code = torch.where(q < 2, q * 2, torch.where(q < 4, q + 2, q / 2 + 4)).to(torch.uint8)
    code = code | ((g < 0) & (code > 0)).to(torch.uint8) * 8
    return code.flatten(-2), (e + 127).to(torch.uint8)


def _pack(k, v):
    """Pages [P, bytes] of fp32 keys and values [P, heads, page, D]. A block of 16 tokens of one head holds the
    keys' codes token by token, the values' codes as [4 quads of tokens][16 parts of D][4 tokens][part], then
    both's scales as [group][token]; codes two to a byte, the first in the low half."""
    P, H, T, D = k.shape
    kc, ks = _codes(k)
    vc, vs = _codes(v)
    kc = (kc[..., 0::2] | kc[..., 1::2] << 4).reshape(P, H, T // 16, 8 * D)
    vc = (vc[..., 0::2] | vc[..., 1::2] << 4).reshape(P, H, T // 16, 4, 4, 16, D // 32)
    vc = vc.transpose(4, 5).reshape(P, H, T // 16, 8 * D)
    ks = ks.reshape(P, H, T // 16, 16, D // 32).transpose(3, 4).reshape(P, H, T // 16, D // 2)
    vs = vs.reshape(P, H, T // 16, 16, D // 32).transpose(3, 4).reshape(P, H, T // 16, D // 2)
    return torch.cat([kc, vc, ks, vs], -1).reshape(P, -1)


def _unpack(pages, H, T, D):
    """fp32 keys and values [..., heads, page, D] of pages [..., bytes]."""
    lead = pages.shape[:-1]
    b = pages.reshape(*lead, H, T // 16, 17 * D)
    kc, vc, ks, vs = b.split([8 * D, 8 * D, D // 2, D // 2], -1)
    vc = vc.reshape(*lead, H, T // 16, 4, 16, 4, D // 32).transpose(-3, -2)
    return [_values(c.reshape(*lead, H, T, D // 2), s.reshape(*lead, H, T // 16, D // 32, 16)) for c, s in ((kc, ks), (vc, vs))]


def _values(codes, scales):
    grid = torch.tensor(GRID + tuple(-x for x in GRID), device=codes.device)
    # one look-up for a byte: two values
    pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], -1)
    x = pairs[codes.to(torch.int32)].flatten(-2)
    s = torch.ldexp(torch.ones((), device=codes.device), scales.to(torch.int32) - 127)
    s = torch.where(scales == 255, math.nan, s)
    s = s.transpose(-1, -2).reshape(*codes.shape[:-1], -1, 1)
    return (x.unflatten(-1, (-1, 32)) * s).flatten(-2)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 17)
    lens, rows = _lens(c)
    H, D, T, L = c["kv_heads"], c["d"], c["page"], c["layers"]
    counts = [_pages_of(n, T) for n in lens]
    slots = c["sessions"] + c["children"]
    widest = max(counts) + _pages_of(c["rows"], T) + 1
    live = sum(counts)
    # free pages among the live ones: what is being grown takes them
    spare = slots * (1 + _pages_of(c["rows"], T)) + 8
    total = max(c["pages"], live if c["path"] == "compact" else live + spare)
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)[:live].cpu()
    table = torch.full((slots, widest), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(counts):
        table[s, :n] = order[at:at + n]
        at += n
    refs = torch.zeros(total, dtype=torch.int32)
    refs[order.long()] = 1
    held = torch.zeros(total, dtype=torch.int32)  # tokens in each page
    for s, n in enumerate(counts):
        if n:
            held[table[s, :n].long()] = T
            held[table[s, n - 1].long()] = lens[s] - (n - 1) * T
    pool = torch.empty((L, total, _page_bytes(c)), dtype=torch.uint8, device="cuda")
    if c["path"] in ("turn", "fork", "compact"):
        # what pages hold is moved as it is
        pool.view(torch.int32).random_(-(1 << 31), (1 << 31) - 1, generator=gen)
    else:
        # keys with a few strong channels, as trained models have them
        channel = torch.exp(0.5 * _normal(gen, H, 1, D))
        step = max(1, (1 << 27) // (H * T * D))
        held = held.cuda()
        for a in range(0, total, step):
            n = min(step, total - a)
            p = _pack((_normal(gen, n, H, T, D) * channel).bfloat16().float(), _normal(gen, n, H, T, D).bfloat16().float())
            # past a page's tokens: what an earlier owner left, here the worst of it
            p = p.view(n, H, T // 16, 17 * D)
            late = (torch.arange(T, device="cuda").view(T // 16, 1, 16) >= held[a:a + n].view(n, 1, 1, 1)).unsqueeze(1)
            p[..., 16 * D:].view(n, H, T // 16, D // 16, 16).masked_fill_(late, 255)
            pool[0, a:a + n] = p.view(n, -1)
    slot_lens = torch.tensor(lens + [0] * c["children"], dtype=torch.int32)
    M = c["sessions"] * c["rows"]
    s = {"case": dict(c), "pool": pool, "table": table.cuda(), "lens": slot_lens.cuda(), "refs": refs.cuda(), "max_len": max(lens),
         "rows": torch.tensor(rows, dtype=torch.int32).cuda() if c["ragged_rows"] else None}
    if c["path"] in ("attend", "step"):
        s["q"] = (1.5 * _normal(gen, M, c["q_heads"], D)).bfloat16()
    if c["path"] in ("append", "step"):
        s["k"] = _normal(gen, M, H, D).bfloat16()
        s["v"] = _normal(gen, M, H, D).bfloat16()
    if c["path"] in ("step", "turn"):
        s["kept"] = s["lens"] - c["rows"]
        s["add"] = torch.full_like(s["lens"], c["rows"])
    if c["path"] == "fork":
        per = c["children"] // c["sessions"]
        s["children"] = torch.arange(c["sessions"], slots, dtype=torch.int32).cuda()
        s["parents"] = torch.arange(c["sessions"], dtype=torch.int32).repeat_interleave(per).cuda()
        s["add"] = torch.tensor([0] * c["sessions"] + [c["rows"]] * c["children"], dtype=torch.int32).cuda()
    return s


def _scale(c):
    return 1.0 / math.sqrt(c["d"])


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2607_13093_amd as sph

    c = s["case"]
    cache = s.get("cache")
    if cache is None:  # the handle that a program keeps
        cache = s["cache"] = sph.KvCache(s["pool"], s["table"], s["lens"], s["refs"], c["kv_heads"], c["d"], c["page"])
    path, rows = c["path"], c["rows"]
    if path == "attend":
        out, lse = sph.kv_attend(cache, 0, s["q"], rows, _scale(c), rows=s["rows"], window=c["window"], max_len=s["max_len"],
                                 want_lse=True)
        return {"out": out, "lse": lse}
    if path == "append":
        sph.kv_append(cache, 0, s["k"], s["v"], rows, rows=s["rows"])
        k, v = sph.kv_read(cache, 0, rows, rows=s["rows"])
        return {"k": k, "v": v}
    if path == "compact":
        if "to" not in s:  # the tables before are kept, so that a pass can be repeated
            s["to"] = torch.empty_like(s["table"]), torch.empty_like(s["refs"])
        table, refs, live = sph.pages_compact(cache, out=s["to"])
        return {"table": table, "refs": refs, "live": live, "pool": s["pool"]}
    if path == "fork":
        sph.pages_fork(cache, s["parents"], s["children"])
        status = sph.pages_grow(cache, s["add"])
        return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status, "pool": s["pool"]}
    sph.pages_trim(cache, s["kept"])
    status = sph.pages_grow(cache, s["add"])
    if path == "turn":
        return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status}
    sph.kv_append(cache, 0, s["k"], s["v"], rows)
    out, lse = sph.kv_attend(cache, 0, s["q"], rows, _scale(c), window=c["window"], max_len=s["max_len"], want_lse=True)
    return {"out": out, "lse": lse, "table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status}


def _run_plain(s):
    c = s["case"]
    path = c["path"]
    if path == "attend":
        return _attend(s)
    if path == "append":
        _append(s)
        return _read(s)
    if path == "compact":
        return _compact(s)
    if path == "fork":
        _fork(s)
        status = _grow(s)
        return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status, "pool": s["pool"]}
    _trim(s, s["kept"])
    status = _grow(s)
    if path == "turn":
        return {"table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status}
    _append(s)
    return {**_attend(s), "table": s["table"], "lens": s["lens"], "refs": s["refs"], "status": status}


def _attend(s):
    c = s["case"]
    S, R, H, D, T, Q = c["sessions"], c["rows"], c["kv_heads"], c["d"], c["page"], c["q_heads"]
    lens = s["lens"][:S].long()
    wide = _pages_of(s["max_len"], T)
    pages = s["pool"][0][s["table"][:S, :wide].clamp(min=0).long()]
    k, v = _unpack(pages, H, T, D)                                     # [S, wide, H, T, D]
    k = k.transpose(1, 2).reshape(S, H, wide * T, D)
    v = v.transpose(1, 2).reshape(S, H, wide * T, D)
    j = torch.arange(wide * T, device=k.device)
    v.masked_fill_((j >= lens.view(S, 1, 1)).unsqueeze(-1), 0.0)       # what lies past the end is anything
    rows = s["rows"].long() if s["rows"] is not None else torch.full_like(lens, R)
    r = torch.arange(R, device=k.device)
    pos = (lens - rows).view(S, 1) + r
    pos = torch.where(r < rows.view(S, 1), pos, -1)
    q = s["q"].float().view(S, R, H, Q // H, D).permute(0, 2, 3, 1, 4).reshape(S, H, -1, D)
    x = torch.matmul(q * _scale(c), k.transpose(-1, -2))
    see = (j <= pos.unsqueeze(-1)) & (j > pos.unsqueeze(-1) - c["window"] if c["window"] else True)   # [S, R, n]
    x = x.view(S, H, Q // H, R, -1).masked_fill_(~see.view(S, 1, 1, R, -1), -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top.clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(S, H, -1, x.shape[-1]), v).view(S, H, Q // H, R, D) / total.clamp(min=1e-30)
    lse = (top + total.log()).squeeze(-1)
    return {"out": o.permute(0, 3, 1, 2, 4).reshape(S * R, Q, D).to(torch.bfloat16),
            "lse": lse.permute(0, 3, 1, 2).reshape(S * R, Q)}


def _places(s):
    """Where each row of the windows lies: first byte of its block of 16 tokens for every head [M, heads], its
    place in the block, and whether it is a row at all."""
    c = s["case"]
    S, R, H, D, T = c["sessions"], c["rows"], c["kv_heads"], c["d"], c["page"]
    lens = s["lens"][:S].long()
    rows = s["rows"].long() if s["rows"] is not None else torch.full_like(lens, R)
    r = torch.arange(R, device=lens.device)
    pos = ((lens - rows).view(S, 1) + r).clamp(min=0)
    page = s["table"][:S].long().gather(1, pos // T).view(-1, 1)
    pos = pos.view(-1, 1)
    heads = torch.arange(H, device=lens.device)
    block = ((page * H + heads) * (T // 16) + pos % T // 16) * (17 * D)
    return block, pos % 16, (r < rows.view(S, 1)).reshape(-1)


def _bytes_of(s):
    """Byte addresses of each row's keys' codes, values' codes, keys' scales and values' scales, [M, heads, n]."""
    D = s["case"]["d"]
    block, tok, valid = _places(s)
    block, tok = block.unsqueeze(-1), tok.unsqueeze(-1)
    i = torch.arange(D // 2, device=block.device)
    g = torch.arange(D // 32, device=block.device)
    kc = block + tok * (D // 2) + i
    part = D // 32
    vc = block + 8 * D + ((tok // 4 * 16 + i // part) * 4 + tok % 4) * part + i % part
    ks = block + 16 * D + g * 16 + tok
    return (kc, vc, ks, ks + D // 2), valid


def _append(s):
    flat = s["pool"][0].view(-1)
    places, valid = _bytes_of(s)
    (kc, ks), (vc, vs) = _codes(s["k"].float()), _codes(s["v"].float())
    data = (kc[..., 0::2] | kc[..., 1::2] << 4, vc[..., 0::2] | vc[..., 1::2] << 4, ks, vs)
    for at, x in zip(places, data):
        flat[at[valid]] = x[valid]


def _read(s):
    flat = s["pool"][0].view(-1)
    (kc, vc, ks, vs), valid = _bytes_of(s)
    k, v = [_values(flat[a], flat[b].unsqueeze(-1)) for a, b in ((kc, ks), (vc, vs))]
    return {n: x.masked_fill(~valid.view(-1, 1, 1), 0.0).to(torch.bfloat16) for n, x in (("k", k), ("v", v))}


def _columns(s):
    return torch.arange(s["table"].shape[1], device=s["table"].device)


def _up(n, page):
    return (n + page - 1) // page


def _count(refs, pages, by):
    refs.index_add_(0, pages.long(), torch.full_like(pages, by))


def _trim(s, kept):
    T = s["case"]["page"]
    now = s["lens"]
    new = torch.minimum(now, kept.clamp(min=0))
    col = _columns(s)
    gone = (col >= _up(new, T).unsqueeze(1)) & (col < _up(now, T).unsqueeze(1))
    _count(s["refs"], s["table"][gone], -1)
    s["table"].masked_fill_(gone, -1)
    now.copy_(new)


def _grow(s):
    T = s["case"]["page"]
    table, refs, now = s["table"], s["refs"], s["lens"]
    new = now + s["add"]
    have, want = _up(now, T), _up(new, T)
    col = _columns(s)
    last = table.gather(1, (now // T).clamp(max=table.shape[1] - 1).long().unsqueeze(1)).squeeze(1)
    shared = (now % T > 0) & (s["add"] > 0) & (refs[last.clamp(min=0).long()] > 1)
    take = (col >= have.unsqueeze(1)) & (col < want.unsqueeze(1)) | shared.unsqueeze(1) & (col == (now // T).unsqueeze(1))
    free = torch.nonzero(refs == 0).squeeze(1).to(torch.int32)
    need = int(take.sum())
    status = torch.tensor([max(0, need - free.numel()), int((want > table.shape[1]).sum())], dtype=torch.int32, device=table.device)
    if int(status.sum()):
        return status
    table[take] = free[:need]
    refs[free[:need].long()] = 1
    source, copy = last[shared].long(), table.gather(1, (now // T).clamp(max=table.shape[1] - 1).long().unsqueeze(1)).squeeze(1)[shared].long()
    _count(refs, last[shared], -1)
    s["pool"][:, copy] = s["pool"][:, source]
    now.copy_(new)
    return status


def _fork(s):
    T = s["case"]["page"]
    table, refs, lens = s["table"], s["refs"], s["lens"]
    p, ch = s["parents"].long(), s["children"].long()
    col = _columns(s)
    old = table[ch][col < _up(lens[ch], T).unsqueeze(1)]
    _count(refs, old, -1)
    mine = col < _up(lens[p], T).unsqueeze(1)
    rows = torch.where(mine, table[p], -1)
    _count(refs, rows[mine], 1)
    table[ch] = rows
    lens[ch] = lens[p]


def _compact(s):
    table, refs, pool = s["table"], s["refs"], s["pool"]
    n = refs.numel()
    live = int((refs > 0).sum())
    holes = torch.nonzero(refs[:live] == 0).squeeze(1)
    movers = torch.nonzero(refs[live:] > 0).squeeze(1) + live
    to = torch.arange(n, dtype=torch.int32, device=refs.device)
    to[movers] = holes.to(torch.int32)
    new = refs.clone()
    new[holes] = refs[movers]
    new[live:] = 0
    pool[:, holes] = pool[:, movers]
    return {"table": torch.where(table >= 0, to[table.clamp(min=0).long()], table), "refs": new,
            "live": torch.tensor([live], dtype=torch.int32, device=refs.device), "pool": pool}


# ---------------------------------------------------------------------------
# the same from the definition, in 64 bits
# ---------------------------------------------------------------------------

def _nearest(x):
    """The 64-bit values that the cache holds for vectors x [n, D]: each 32 share 2^e, the least e for which the
    largest still rounds to at most 6 of the E2M1 steps."""
    g = x.view(x.shape[0], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -127.0)
    for k in range(-127, 128):  # up while the top is at least 7 steps
        e = torch.where((e == k) & (top >= 7 * 2.0 ** k), e + 1, e)
    a = g.abs() / 2.0 ** e
    steps = [(a > 0.25), (a >= 0.75), (a > 1.25), (a >= 1.75), (a > 2.5), (a >= 3.5), (a > 5.0)]
    sizes = (0.5, 0.5, 0.5, 0.5, 1.0, 1.0, 2.0)
    y = sum(m.double() * h for m, h in zip(steps, sizes)) * 2.0 ** e
    return (torch.where(g < 0, -y, y)).view(x.shape)


def _token(pool, page, head, tok, c):
    """64-bit key and value vectors [n, D] of tokens: 1-D tensors of page, head and place in the page."""
    H, D, T = c["kv_heads"], c["d"], c["page"]
    base = ((page * H + head) * (T // 16) + tok // 16) * 17 * D
    t = tok % 16
    d = torch.arange(D, device=pool.device)
    flat = pool.reshape(-1)
    part = D // 16
    key = base[:, None] + t[:, None] * (D // 2) + d // 2
    val = base[:, None] + 8 * D + (t[:, None] // 4 * 16 + d // part) * (D // 8) + t[:, None] % 4 * (D // 32) + d % part // 2
    scl = base[:, None] + 16 * D + d // 32 * 16 + t[:, None]
    out = []
    for at, sc in ((key, scl), (val, scl + D // 2)):
        code = torch.bitwise_right_shift(flat[at].int(), (d % 2 * 4).int()) & 15
        mag, sign = code & 7, code >> 3
        # E2M1: two exponent bits, one mantissa bit, subnormal below 1
        y = torch.where(mag < 2, mag * 0.5, (1 + (mag & 1) * 0.5) * 2.0 ** ((mag >> 1) - 1).double())
        out.append(torch.where(sign > 0, -y, y).double() * 2.0 ** (flat[sc].double() - 127))
    return out


def exact(case, seed):
    c = case
    if c["path"] not in ("attend", "append", "step"):
        return None
    s = prepare(c, seed)
    lens, rows = _lens(c)
    R, H, D, T, Q = c["rows"], c["kv_heads"], c["d"], c["page"], c["q_heads"]
    dev = s["pool"].device
    if c["path"] == "append":
        valid = torch.zeros(c["sessions"], R, 1, dtype=torch.float64, device=dev)
        for i, r in enumerate(rows):
            valid[i, :r] = 1.0
        # as fp64: a code's value, 0 where there is no row
        return {n: (_nearest(s[n].double().view(-1, D)).view(c["sessions"], R, -1) * valid).view(-1, H, D) for n in ("k", "v")}
    out = torch.zeros(c["sessions"], R, Q, D, dtype=torch.float64, device=dev)
    lse = torch.full((c["sessions"], R, Q), -math.inf, dtype=torch.float64, device=dev)
    G = Q // H
    for i, (n, r) in enumerate(zip(lens, rows)):
        first = max(0, n - r - c["window"] + 1) if c["window"] else 0
        pos = torch.arange(n - r, n, device=dev)
        j = torch.arange(first, n, device=dev)
        page = s["table"][i].long()[j // T]
        for h in range(H):
            k, v = _token(s["pool"][0], page, torch.full_like(j, h), j % T, c)
            if c["path"] == "step":
                k[j >= n - r] = _nearest(s["k"].view(-1, R, H, D)[i, :, h].double())
                v[j >= n - r] = _nearest(s["v"].view(-1, R, H, D)[i, :, h].double())
            for a in range(0, r, 1024):
                b = min(r, a + 1024)
                q = s["q"].view(-1, R, Q, D)[i, a:b, h * G:(h + 1) * G].double()
                x = q.reshape(-1, D) @ k.T / math.sqrt(D)
                see = (j[None] <= pos[a:b, None]) & ((j[None] > pos[a:b, None] - c["window"]) if c["window"] else True)
                x = x.view(b - a, G, -1).masked_fill(~see[:, None], -math.inf)
                top = x.amax(-1, keepdim=True).clamp(min=-1e300)
                p = (x - top).exp()
                z = p.sum(-1, keepdim=True)
                out[i, a:b, h * G:(h + 1) * G] = ((p.view(-1, p.shape[-1]) @ v).view(b - a, G, D) / z.clamp(min=1e-300))
                lse[i, a:b, h * G:(h + 1) * G] = (top + z.log()).squeeze(-1)
    found = {"out": out.view(-1, Q, D), "lse": lse.view(-1, Q)}
    return {**found, "table": None, "lens": None, "refs": None, "status": None} if c["path"] == "step" else found
