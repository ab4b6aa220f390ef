"""Page growth at the ends of its argument range."""

import pytest
import torch

import paper_2607_13093_amd as sph

from kv_build import host
from test_gpu_pages import ints, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages", [64, 140000])    # by one workgroup, by several
@pytest.mark.parametrize("slots,each,lacking", [
    (33, 1 << 30, (1 << 31) - 1),                    # 2^31 + 2^26 pages and more: a negative number in 32 bits
    (64, 1 << 30, (1 << 31) - 1),                    # 2^32: none
    (65, 1 << 30, (1 << 31) - 1),                    # 2^32 + 2^26
    (31, 1 << 30, 31 << 26), (3, 1 << 20, 3 << 16),  # in 32 bits
])
def test_sums_of_pages_past_32_bits(n_pages, slots, each, lacking):
    say("pages lacking", n_pages, slots, each)
    most = each // 16
    # a table of up to 17 GB, of which only what sessions hold is read
    table = torch.empty((slots, most), dtype=torch.int32, device="cuda")
    c = sph.KvCache(torch.empty((1, n_pages, sph.kv_page_bytes(1, 64, 16)), dtype=torch.uint8, device="cuda"), table,
                    torch.zeros(slots, dtype=torch.int32, device="cuda"),
                    torch.zeros(n_pages, dtype=torch.int32, device="cuda"), 1, 64, 16)
    status = sph.pages_grow(c, ints([each] * slots))
    assert host(status).tolist() == [lacking - n_pages, 0]
    assert not bool(c.lens.any()) and not bool(c.refs.any())
    # and what fits is still given out
    table[:, :8] = -1
    status = sph.pages_grow(c, ints([33, 0] + [16] * 20 + [0] * (slots - 22) if slots >= 22 else [33, 0, 16]))
    assert host(status).tolist() == [0, 0]
    n = 3 + (20 if slots >= 22 else 1)
    assert host(c.refs[:n]).tolist() == [1] * n and not bool(c.refs[n:].any())
    assert host(table[0, :3]).tolist() == [0, 1, 2] and host(table[2, :1]).tolist() == [3]
