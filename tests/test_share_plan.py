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


SIZES = [  # kv heads, group, d, sessions, R
    (8, 4, 128, 1, 1), (1, 1, 64, 2, 1), (8, 4, 128, 16, 5), (8, 8, 128, 256, 8), (16, 4, 256, 256, 9),
    (8, 5, 128, 4, 2047), (64, 1, 256, 4, 4095), (64, 1, 256, 3, 1811), (64, 1, 256, 3, 1355), (64, 1, 256, 3, 1084),
    (128, 1, 64, 4, 8191), (16, 4, 256, 4, 4095), (8, 8, 256, 2048, 3), (1, 32, 64, 3, 700), (2, 1, 256, 3, 1 << 23),
    (32768, 1, 128, 2048, 1),
]


@pytest.mark.parametrize("max_len", [0, 1, 300, 9000])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_parts_stay_within_their_bound(case, max_len):
    # 4 d + 8 bytes a row, head and part: at most a GiB, or two parts where those are more
    lib = _lib.load()
    heads, group, d, n, R = SIZES[case]
    c = described(kv_heads=heads, head_dim=d)
    need = lib.sph_kv_attend_shared_workspace(ctypes.addressof(c), heads * group, n, R, max_len)
    part = n * R * heads * group * (4 * d + 8)
    assert 2 * part <= need <= max(1 << 30, 2 * part) + 256
    assert need <= 60 * part + 256
    assert lib.sph_kv_share_bytes(ctypes.addressof(c), heads * group, n, R, max_len) > 0
