"""What a sharing plan and its workspace are sized for, asked without a device."""

import ctypes
from types import SimpleNamespace

import pytest
import torch

from paper_2607_13093_amd import _lib
from paper_2607_13093_amd.api import KvSharePlan


def described(**kw):
    a = dict(pool=4096, layers=1, layer_stride=1 << 40, n_pages=1 << 20, page_stride=1 << 30, table=4096, ld_table=1 << 16,
             max_pages=1 << 16, lens=4096, refs=4096, n_slots=4096, kv_heads=8, head_dim=128, page_tokens=16)
    a.update(kw)
    return _lib.KvCacheStruct(*a.values())


def test_a_plan_is_fixed():
    # a smaller tensor in the buffer's place would be written past its end, by the size of the one before
    struct = described()
    cache = SimpleNamespace(ptr=ctypes.addressof(struct), device=torch.device("cpu"))
    plan = KvSharePlan(cache, 32, 3, 5, None, None, 0, 0)
    assert plan.buffer.numel() == plan.bytes > 0 and plan.workspace_bytes > 0
    for name in ("buffer", "bytes", "workspace_bytes", "cache", "q_heads", "n_sessions", "rows_per_session", "window", "max_len"):
        was = getattr(plan, name)
        with pytest.raises(AttributeError, match=name):
            setattr(plan, name, was)
        assert getattr(plan, name) is was
    plan.rows = plan.slots = torch.zeros(3, dtype=torch.int32)  # those of the next kv_share
