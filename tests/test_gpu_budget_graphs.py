"""A server's step captured into a graph, with all that it does to sessions that share and
forget: growth, the plan, each layer's append, shared attention and weights, and eviction.
Every replay is compared, bit for bit, with the same step run eagerly on a copy of the cache
as it was, between replays that the caller's own work separates."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph

from kv_build import bf16, host
from test_gpu_share import ints, say

pytestmark = pytest.mark.gpu

LAYERS, SLOTS, R = 2, 6, 3


class Step:
    """Inputs, outputs and workspaces of a step at fixed places."""

    def __init__(self, c, group):
        self.c = c
        hq, d, width = c.kv_heads * group, c.head_dim, c.table.shape[1] * c.page_tokens
        self.rows = torch.zeros(SLOTS, dtype=torch.int32, device="cuda")
        self.keep = torch.zeros(SLOTS, dtype=torch.int32, device="cuda")
        self.q = torch.zeros(LAYERS, SLOTS * R, hq, d, dtype=torch.bfloat16, device="cuda")
        self.k = torch.zeros(LAYERS, SLOTS * R, c.kv_heads, d, dtype=torch.bfloat16, device="cuda")
        self.out = [(torch.empty_like(self.q[0]), torch.empty(SLOTS * R, hq, device="cuda")) for _ in range(LAYERS)]
        self.weights = torch.zeros(SLOTS, width, device="cuda")
        self.kept = torch.full((SLOTS, width), -1, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(2, dtype=torch.int32, device="cuda")
        self.hq = hq
        self.plan = sph.kv_share(c, hq, R, rows=self.rows)

    def run(self):
        c = self.c
        sph.pages_grow(c, self.rows, out=self.status)
        sph.kv_share(c, self.hq, R, rows=self.rows, out=self.plan)
        for i in range(LAYERS):
            sph.kv_append(c, i, self.k[i], self.k[i], R, rows=self.rows)
            sph.kv_attend_shared(c, i, self.q[i], self.plan, 0.1, out=self.out[i])
            sph.kv_weigh(c, i, self.q[i], self.out[i][1], R, 0.1, self.weights, rows=self.rows, fresh=i == 0)
        sph.pages_evict(c, self.weights, self.keep, 2, R, out=(self.weights, self.kept))

    def held(self):
        c = self.c
        return [c.pool, c.table, c.lens, c.refs, self.weights, self.kept, self.status, *self.out[0], *self.out[1]]


@pytest.mark.parametrize("heads,group,d,page", [(2, 4, 64, 16), (2, 3, 128, 32), (1, 8, 256, 16)])
def test_steps_captured_and_replayed(heads, group, d, page):
    rng = np.random.default_rng(d)
    c = sph.KvCache.empty(LAYERS, 160, SLOTS, 30, heads, d, page)
    c.pool.fill_(0x11)  # finite codes and scales
    assert host(sph.pages_grow(c, ints([300, 0, 0, 0, 90, 0]))).tolist() == [0, 0]
    sph.pages_fork(c, ints([0, 0, 0]), ints([1, 2, 3]))
    captured = Step(c, group)
    copy = sph.KvCache(c.pool.clone(), c.table.clone(), c.lens.clone(), c.refs.clone(), heads, d, page)
    eager = Step(copy, group)
    captured.keep.fill_(1 << 20)
    say("warm-up", heads, group, d, page)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())  # (the cache is still being filled)
    with torch.cuda.stream(side):
        captured.run()  # of no rows: changes nothing that is held
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    torch.cuda.synchronize()
    for turn in range(5):
        counts = ints([[3, 1, 2, 0, 3, 1], [1, 1, 1, 1, 1, 1], [3, 3, 3, 3, 3, 3], [0, 2, 1, 3, 0, 2], [2, 0, 0, 1, 3, 3]][turn])
        keep = ints([[1 << 20] * 6, [310, 303, 305, 302, 80, 1], [200] * 6, [290, 289, 400, 1 << 20, 60, 2], [0] * 6][turn])
        q, k = bf16(rng, *captured.q.shape)[0], bf16(rng, *captured.k.shape)[0]
        for s in (captured, eager):
            s.rows.copy_(counts), s.keep.copy_(keep), s.q.copy_(q), s.k.copy_(k), s.kept.fill_(-1)
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        assert host(captured.status).tolist() == [0, 0]
        for i, (a, b) in enumerate(zip(captured.held(), eager.held())):
            assert torch.equal(a, b), (turn, i)
        say("turn", turn, "held", host(c.lens).tolist())
    assert torch.isfinite(captured.weights).all()
