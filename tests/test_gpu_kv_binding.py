"""What the torch binding of the cache takes and gives back."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph

from kv_build import bf16, cache_of, filled, host
from test_gpu_kv import say

pytestmark = pytest.mark.gpu


def test_a_cache_is_fixed():
    # another tensor in an attribute's place would not be the one that calls work on
    rng = np.random.default_rng(1)
    c = cache_of(rng, [20, 5], 2, 64, 16)
    for name in ("pool", "table", "lens", "refs"):
        was = getattr(c, name)
        with pytest.raises(AttributeError, match=name):
            setattr(c, name, was.clone())
        assert getattr(c, name) is was
    for name in ("kv_heads", "head_dim", "page_tokens", "layers", "n_pages", "n_slots", "device", "ptr"):
        with pytest.raises(AttributeError, match=name):
            setattr(c, name, getattr(c, name))
    c.note = 1                                     # what is not the cache's is free
    c.note = 2
    say("in place")
    c.lens.copy_(torch.tensor([3, 4], dtype=torch.int32))
    sph.pages_trim(c, torch.tensor([2, 9], dtype=torch.int32).cuda())
    assert host(c.lens).tolist() == [2, 4]


def test_log_sum_exp_beside_an_output_of_the_caller():
    rng = np.random.default_rng(2)
    c, _, _ = filled(rng, [40, 7], 2, 64, 16)
    q, _ = bf16(rng, 2 * 3, 4, 64)
    want, wl = sph.kv_attend(c, 0, q, 3, 0.1, want_lse=True)
    o = torch.empty_like(q)
    say("lse wanted, none given")
    got, lse = sph.kv_attend(c, 0, q, 3, 0.1, want_lse=True, out=(o, None))
    assert got is o and torch.equal(o, want) and torch.equal(lse, wl)
    say("not wanted, none given; given")
    assert sph.kv_attend(c, 0, q, 3, 0.1, out=(o, None))[1] is None
    mine = torch.empty_like(wl)
    assert sph.kv_attend(c, 0, q, 3, 0.1, out=(o, mine))[1] is mine and torch.equal(mine, wl)


def test_workspaces_off_the_cache_s_device_are_refused():
    # a kernel would write to host memory
    rng = np.random.default_rng(3)
    c, _, _ = filled(rng, [3000], 1, 128, 16)
    q, _ = bf16(rng, 1, 8, 128)
    want, _ = sph.kv_attend(c, 0, q, 1, 0.1)
    need = sph.kv_attend_workspace(c, 8, 1, 1)
    add = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert need > 0
    big = torch.empty(1 << 22, dtype=torch.uint8)
    for bad, what in ((big, "on cpu"), (big.cuda()[::2], "contiguous")):
        with pytest.raises(ValueError, match=what):
            sph.kv_attend(c, 0, q, 1, 0.1, workspace=bad)
        with pytest.raises(ValueError, match=what):
            sph.pages_grow(c, add, workspace=bad)
        with pytest.raises(ValueError, match=what):
            sph.pages_compact(c, workspace=bad)
    say("workspaces of other types, in bytes")
    ws = torch.empty((need + 3) // 4, dtype=torch.float32, device="cuda")
    assert torch.equal(sph.kv_attend(c, 0, q, 1, 0.1, workspace=ws)[0], want)
    with pytest.raises(sph.SphError, match="workspace"):
        sph.kv_attend(c, 0, q, 1, 0.1, workspace=ws[:-1])


def test_workspaces_begin_at_any_16_bytes():
    rng = np.random.default_rng(4)
    c, _, _ = filled(rng, [3000, 40], 1, 128, 16)
    q, _ = bf16(rng, 2, 8, 128)
    want, wl = sph.kv_attend(c, 0, q, 1, 0.1, want_lse=True)
    buf = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    assert buf.data_ptr() % 256 == 0 and sph.kv_attend_workspace(c, 8, 2, 1) > 0
    table, refs, lens = c.table.clone(), c.refs.clone(), c.lens.clone()
    add = torch.tensor([20, 1], dtype=torch.int32).cuda()
    kept = torch.tensor([3000, 40], dtype=torch.int32).cuda()
    for at in (16, 240):
        say("workspace at", at)
        got, lse = sph.kv_attend(c, 0, q, 1, 0.1, want_lse=True, workspace=buf[at:])
        assert torch.equal(got, want) and torch.equal(lse, wl)
        assert host(sph.pages_grow(c, add, workspace=buf[at:])).tolist() == [0, 0]
        assert host(c.lens).tolist() == [3020, 41]
        sph.pages_trim(c, kept)
        assert torch.equal(c.table, table) and torch.equal(c.refs, refs) and torch.equal(c.lens, lens)
        out = torch.empty_like(table), torch.empty_like(refs)
        live = sph.pages_compact(c, out=out, workspace=buf[at:])[2]
        assert int(live) == int((refs > 0).sum()) == int((out[1] > 0).sum())
        c.table.copy_(out[0]), c.refs.copy_(out[1])
        assert torch.equal(sph.kv_attend(c, 0, q, 1, 0.1)[0], want)
        table, refs = c.table.clone(), c.refs.clone()
    with pytest.raises(sph.SphError, match="16"):
        sph.kv_attend(c, 0, q, 1, 0.1, workspace=buf[8:])
