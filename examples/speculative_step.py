"""Speculative decoding with the paged 4-bit cache and the split vocabulary head.

A toy decoder of one attention layer with random weights answers prompts. Each step
runs a window of R rows a session (its last token and R - 1 drafts): pages for the
window, its keys and values into the cache, attention over it, the cloud's and the
endpoint's half of the head, verification; then the rows of rejected drafts are given
back. Between steps one session is branched into others, which share its pages until
they write, and the pool is compacted.

    python examples/speculative_step.py [--steps 4] [--sessions 4]
"""

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_13093_amd as sph  # noqa: E402


class ToyDecoder:
    """Embedding, one attention layer, the head split in two."""

    def __init__(self, vocab=8192, d=512, d_end=64, q_heads=8, kv_heads=2, head_dim=64, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") / shape[-1] ** 0.5).to(torch.bfloat16)

        self.d, self.d_end, self.q_heads, self.kv_heads, self.head_dim = d, d_end, q_heads, kv_heads, head_dim
        self.embed = torch.randn(vocab, d, generator=g, device="cuda").to(torch.bfloat16)
        self.qkv = weight((q_heads + 2 * kv_heads) * head_dim, d)
        self.out = weight(d, q_heads * head_dim)
        self.w_cloud, self.w_end = weight(vocab, d - d_end), weight(vocab, d_end)

    def layer(self, cache, tokens, rows_per_session, rows=None, slots=None):
        """Hidden rows of tokens [sessions * R]; their keys and values join the cache."""
        x = self.embed[tokens.long()]
        y = (x @ self.qkv.T).view(-1, self.q_heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = y.split([self.q_heads, self.kv_heads, self.kv_heads], dim=1)
        sph.kv_append(cache, 0, k, v, rows_per_session, rows=rows, slots=slots)
        o, _ = sph.kv_attend(cache, 0, q, rows_per_session, self.head_dim ** -0.5, rows=rows, slots=slots)
        return x + o.reshape(-1, self.q_heads * self.head_dim) @ self.out.T


def step(model, cache, subset, last, drafts):
    """One window of every slot: last token [n] and drafts [n, k]. Returns the rows'
    tokens [n, k + 1] and the accepted drafts [n]; the cache ends with what is kept."""
    n, k = drafts.shape
    R = k + 1
    status = sph.pages_grow(cache, torch.full_like(cache.lens, R))
    tokens = torch.cat([last.view(n, 1), drafts], 1).reshape(-1)
    h = model.layer(cache, tokens, R)
    q, scale, _ = sph.cloud_partial(h[:, model.d_end:], model.w_cloud, subset, 30.0)
    out, accept, _ = sph.fuse_verify(q, scale, h[:, :model.d_end], model.w_end, subset, n, R, drafts.contiguous())
    # rows past the accepted drafts leave the cache; the token after them is the next step's
    sph.pages_trim(cache, cache.lens - (k - accept))
    return out.view(n, R), accept, status


def run(sessions=4, steps=4, k=3, page=16, seed=0, draft=None, say=print):
    """draft(answers, k) -> int32 [slots, k]: a draft model; without one, drafts are what the head
    said for the rows after the accepted ones."""
    model = ToyDecoder()
    subset = sph.Subset(torch.arange(0, 8192, 2).numpy(), vocab=8192)
    longest = 200
    slots, max_pages = sessions + 2, longest // page + steps + 2
    cache = sph.KvCache.empty(1, slots * max_pages, slots, max_pages, model.kv_heads, model.head_dim, page)
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(5, longest, (sessions,), generator=g).tolist()

    # prompts of different lengths, in one call
    rows = torch.tensor(lens + [0] * (slots - sessions), dtype=torch.int32).cuda()
    sph.pages_grow(cache, rows)
    prompt = torch.randint(0, 8192, (slots * longest,), generator=g).cuda()
    h = model.layer(cache, prompt, longest, rows=rows)
    # the last session is branched twice: the branches share its pages
    branches = torch.arange(sessions, slots, dtype=torch.int32).cuda()
    sph.pages_fork(cache, torch.full_like(branches, sessions - 1), branches)
    at = torch.tensor(lens + [lens[-1]] * 2).cuda() - 1
    at = at + longest * torch.tensor(list(range(sessions)) + [sessions - 1] * 2).cuda()
    hl = h[at].contiguous()
    q, s, _ = sph.cloud_partial(hl[:, model.d_end:], model.w_cloud, subset, 30.0)
    last, _, _ = sph.fuse_verify(q, s, hl[:, :model.d_end], model.w_end, subset, slots, 1, None)
    last[sessions:] = torch.tensor([2, 4], dtype=torch.int32).cuda()  # branches differ from here on

    answers = [[int(t)] for t in last]
    guess = torch.randint(0, 4096, (slots, k), generator=g).to(torch.int32).cuda() * 2
    for i in range(steps):
        if draft is not None:
            guess = draft(answers, k)
        out, accept, status = step(model, cache, subset, last, guess)
        assert status.tolist() == [0, 0], "the pool is too small"
        took = accept.tolist()
        for s in range(slots):
            answers[s] += guess[s, :took[s]].tolist() + [int(out[s, took[s]])]
        last = out.gather(1, accept.long().view(-1, 1)).view(-1)
        guess = out.roll(-1, 1)[:, :k].contiguous()
        say(f"step {i}: accepted {took}, cached {cache.lens.tolist()}, pages in use {int((cache.refs > 0).sum())}")
        if i % 2 == 1:
            table, refs, live = sph.pages_compact(cache)
            say(f"        compacted to {int(live)} pages")
    return cache, answers


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--sessions", type=int, default=4)
    ap.add_argument("--steps", type=int, default=4)
    a = ap.parse_args()
    _, answers = run(a.sessions, a.steps)
    for s, t in enumerate(answers):
        print(f"session {s}: {t}")


if __name__ == "__main__":
    main()
