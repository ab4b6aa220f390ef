"""Pins of the oracle of token weights and eviction: closed forms and hand-worked slots."""

import math

import numpy as np

from oracle import kv_budget as B
from oracle import kv_cache as O


def test_choose_by_hand():
    w = [5.0, 1.0, 3.0, 3.0, 9.0, 0.0, 3.0, 2.0]
    assert B.choose(w, 8, 4, 0, 0) == [0, 2, 3, 4]                # ties go to the first
    assert B.choose(w, 8, 5, 0, 0) == [0, 2, 3, 4, 6]
    assert B.choose(w, 8, 4, 2, 2) == [0, 1, 6, 7]                # what is certain fills it
    assert B.choose(w, 8, 1, 2, 2) == [0, 1, 6, 7]                # and may be more than it
    assert B.choose(w, 8, 8, 0, 0) == list(range(8)) == B.choose(w, 8, 100, 1, 1)
    assert B.choose(w, 3, 1, 0, 0) == [0] and B.choose(w, 0, 3, 2, 2) == []
    assert B.choose(w, 8, -4, 0, 0) == [] and B.choose(w, 8, 0, 0, 50) == list(range(8))
    odd = [math.nan, -math.inf, -0.0, 0.0, math.inf, math.nan, 1e-45]
    assert B.choose(odd, 7, 1, 0, 0) == [4] and B.choose(odd, 7, 2, 0, 0) == [4, 6]
    assert B.choose(odd, 7, 3, 0, 0) == [2, 4, 6]                 # zeros of both signs are equal
    assert B.choose(odd, 7, 5, 0, 0) == [1, 2, 3, 4, 6] and B.choose(odd, 7, 6, 0, 0) == [0, 1, 2, 3, 4, 6]


def test_evict_leaves_shared_pages():
    table = np.array([[0, 1, 2, -1], [0, 1, 3, 4]])
    refs = np.array([2, 2, 1, 1, 1, 0])
    w = np.zeros((2, 16))
    w[0, 10] = w[1, 13] = 1
    kept, t, lens, r = B.evict(table, np.array([11, 16]), refs, w, [0, 10], 0, 0, 4)
    assert kept == [list(range(8)), list(range(9)) + [13]]
    assert lens.tolist() == [8, 10] and r.tolist() == [2, 2, 0, 1, 0, 0]
    assert t.tolist() == [[0, 1, -1, -1], [0, 1, 3, -1]]
    assert table[0, 2] == 2 and refs[2] == 1                      # inputs as they were


def test_weights_of_a_row_sum_to_one():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((3, 4, 32)), rng.standard_normal((9, 2, 32))
    for window in (0, 4):
        _, lse, _, _ = O.attend(q, k, k, 0.3, 3, window)
        total, slack = B.weigh(q, k, lse, 0.3, 3, window)
        assert abs(total.sum() - 12) < 1e-12 and (slack >= total).all()
        assert (total[:3] > 0).all() if window == 0 else (total[:3] == 0).all()
    # equal keys share a row's weight
    flat = np.ones((5, 1, 32))
    _, lse, _, _ = O.attend(q[:1, :1], flat, flat, 0.3, 1)
    np.testing.assert_allclose(B.weigh(q[:1, :1], flat, lse, 0.3, 1)[0], 0.2, rtol=1e-12)
    # a row without a log-sum-exp adds nothing, nor do rows past the session's
    assert not B.weigh(q, k, np.full((3, 4), -np.inf), 0.3, 3)[0].any() and not B.weigh(q, k, lse, 0.3, 0)[0].any()
