"""Pins of the cache oracle that do not go by its own code."""

import numpy as np
import torch

from oracle import kv_cache as O


def test_quantize_hand_worked():
    x = np.zeros(64)
    x[:8] = [6.0, -3.0, 1.25, 0.25, 0.75, 2.5, -5.0, 0.24]     # e = 0: ties to even codes
    x[32:36] = [7.0, 6.9, 3.0, 1.0]                             # 7 would round past 6: e = 1
    y = O.quantize(x)
    np.testing.assert_array_equal(y[:8], [6.0, -3.0, 1.0, 0.0, 1.0, 2.0, -4.0, 0.0])
    np.testing.assert_array_equal(y[32:36], [8.0, 6.0, 3.0, 1.0])
    assert not y[8:32].any() and not y[36:].any()


def test_quantize_rounds_to_the_grid_of_its_group():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((200, 32)) * np.exp(rng.uniform(-20, 20, (200, 1)))
    y = O.quantize(x)
    top = np.abs(x).max(1)
    # the shared step: the largest lies in [3.5, 7) steps, so it is off by at most one
    e = np.floor(np.log2(top)) - 2
    e = np.where(top / 2.0 ** e >= 7, e + 1, e)
    a = np.abs(y) / 2.0 ** e[:, None]
    assert np.isin(a, O.E2M1).all()
    assert (top / 2.0 ** e >= 3.5).all() and (top / 2.0 ** e < 7).all()
    # nearest: no grid value is nearer
    for g in O.E2M1:
        assert (np.abs(np.abs(x) / 2.0 ** e[:, None] - a) <= np.abs(np.abs(x) / 2.0 ** e[:, None] - g) + 1e-12).all()
    np.testing.assert_array_equal(O.quantize(y), y)             # idempotent


def test_attend_against_torch():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((3, 4, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    out, lse, mag, _ = O.attend(q, k, v, 0.2, 3)
    t = [torch.tensor(a) for a in (q, k, v)]
    mask = torch.ones(3, 9, dtype=torch.bool).tril(6)
    ref = torch.nn.functional.scaled_dot_product_attention(
        t[0].transpose(0, 1), t[1].transpose(0, 1).repeat_interleave(2, 0),
        t[2].transpose(0, 1).repeat_interleave(2, 0), attn_mask=mask, scale=0.2).transpose(0, 1)
    np.testing.assert_allclose(out, ref.numpy(), rtol=0, atol=1e-12)
    assert (mag >= np.abs(out) - 1e-12).all() and np.isfinite(lse).all()
    # one token: its value; a window of one: the row's own token
    one = O.attend(q[:1], k[:1], v[:1], 0.2, 1)
    np.testing.assert_array_equal(one[0][0, 0], v[0, 0])
    np.testing.assert_allclose(O.attend(q, k, v, 0.2, 3, window=1)[0][:, 3], v[6:, 1], rtol=0, atol=0)
    # more rows than tokens: the first see nothing
    none = O.attend(q, k[:2], v[:2], 0.2, 3)
    assert not none[0][0].any() and np.isneginf(none[1][0]).all() and np.isfinite(none[1][1:]).all()


def test_pages_by_hand():
    p = O.Pages(n_pages=6, n_slots=3, max_pages=3, page=4)
    assert p.grow([5, 0, 4]) == (0, 0)
    np.testing.assert_array_equal(p.table, [[0, 1, -1], [-1] * 3, [2, -1, -1]])
    p.fork([0], [1])
    np.testing.assert_array_equal(p.refs, [2, 2, 1, 0, 0, 0])
    assert p.grow([0, 4, 0]) == (0, 0)             # the shared page 1 is copied to 3, then 4 is new
    np.testing.assert_array_equal(p.table[1], [0, 3, 4])
    np.testing.assert_array_equal(p.refs, [2, 1, 1, 1, 1, 0])
    assert p.content == [0, 1, 2, 1, 4, 5] and list(p.lens) == [5, 9, 4]
    assert p.grow([4, 0, 4]) == (1, 0) and p.grow([0, 4, 0]) == (0, 1)   # nothing changes
    assert list(p.lens) == [5, 9, 4]
    p.trim([0, 9, 1])
    np.testing.assert_array_equal(p.refs, [1, 0, 1, 1, 1, 0])
    assert p.compact() == 4                        # page 4 moves to 1
    np.testing.assert_array_equal(p.table, [[-1] * 3, [0, 3, 1], [2, -1, -1]])
    np.testing.assert_array_equal(p.refs, [1, 1, 1, 1, 0, 0])
