"""Token weights on the GPU by the number of rows of a head: each number of row tiles that
the kernel for few rows is built for, and the first that the one for many takes, against
the 64-bit oracle within the bound of test_gpu_weigh.py."""

import numpy as np
import pytest
import torch

import paper_2607_13093_amd as sph
from oracle import kv_budget as B
from oracle import kv_cache as O

from kv_build import bf16, filled, host
from test_gpu_weigh import ints, say, within

pytestmark = pytest.mark.gpu


# (rows of a session, query heads of a key/value head): 16, 17 to 32, 33 to 64 rows of a head, and 72
ROWS = [(4, 4), (6, 4), (8, 4), (11, 3), (8, 8), (9, 8)]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("R,group", ROWS)
@pytest.mark.parametrize("window", [0, 70])
def test_tiles_of_rows(d, R, group, window):
    say("tiles", d, R, group, window)
    rng = np.random.default_rng(d + R * group)
    # tokens that end inside a tile of 32, in the first and in a later wave and workgroup; fewer than rows; none
    lens, heads, page = [700, 261, 33, 3, 0, 512], 2, 32
    rows = [R, R - 1, R, R, 1, 1]
    c, keys, _ = filled(rng, lens, heads, d, page)
    n, scale, width = len(lens), d ** -0.5, c.table.shape[1] * page
    for pad in (0, 3):  # with 3, rows of q are off 16 bytes
        q, q64 = bf16(rng, n * R, heads * group, d + pad)
        q, q64 = q[..., pad:], q64[..., pad:].reshape(n, R, heads * group, d)
        lse = np.stack([O.attend(q64[s], keys[s], keys[s], scale, rows[s], window)[1] for s in range(n)])
        w = rng.random((n, width)).astype(np.float32)
        lse32 = torch.from_numpy(lse.reshape(n * R, -1).astype(np.float32)).cuda()
        for max_len in (0, 1, 700):
            weights = torch.from_numpy(w).cuda()
            sph.kv_weigh(c, 0, q, lse32, R, scale, weights, rows=ints(rows), window=window, max_len=max_len)
            got = host(weights)
            for s in range(n):
                within(got[s, :lens[s]], w[s, :lens[s]].astype(np.float64),
                       *B.weigh(q64[s], keys[s], lse[s], scale, rows[s], window), d, R * heads * group)
                np.testing.assert_array_equal(got[s, lens[s]:], w[s, lens[s]:])
