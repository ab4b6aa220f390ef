"""The example of a speculative decoder runs, and its cache ends as its answers say:
decoding the same tokens one at a time, with no drafts, gives the same answers."""

import os
import sys

import pytest
import torch

import paper_2607_13093_amd as sph

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_speculative_answers_are_those_of_plain_decoding():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import speculative_step as ex
    finally:
        sys.path.pop(0)
    print("[gpu] example: one row a step", flush=True)
    _, slow = ex.run(sessions=3, steps=16, k=0, say=lambda *a: None)
    seen = []

    def draft(answers, k):
        # right for as many drafts as the step's turn says, then wrong ones
        right = [(len(seen) + s) % (k + 1) for s in range(len(answers))]
        seen.append(right)
        return torch.tensor([[slow[s][len(a) + i] if i < right[s] else slow[s][len(a) + i] ^ 2 for i in range(k)]
                             for s, a in enumerate(answers)], dtype=torch.int32).cuda()

    print("[gpu] example: two drafts a step", flush=True)
    lines = []
    cache, fast = ex.run(sessions=3, steps=5, k=2, draft=draft, say=lines.append)
    took = [ln for ln in lines if "accepted" in ln]
    assert [f"accepted {r}" in ln for r, ln in zip(seen, took)] == [True] * 5
    assert len(fast) == len(slow) == 5
    for a, b in zip(fast, slow):
        n = min(len(a), len(b))
        assert n >= 6 and a[:n] == b[:n]
    # the cache holds each prompt and every answered token but the last
    refs = torch.zeros_like(cache.refs)
    held = cache.table[cache.table >= 0].long()
    refs.index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    assert torch.equal(refs, cache.refs)
    assert int((cache.table >= 0).sum()) == int(((cache.lens + 15) // 16).sum())
