"""Pins of the float64 paged-cache and log-probability oracle on cases that can be done by hand."""
import math

import numpy as np

from oracle import paged as OP


def test_rotation_is_a_rotation_by_the_position():
    x = np.array([[1.0, 2.0, 3.0, 4.0]])
    assert np.array_equal(OP.rotate(x, 7, 0), x)
    y = OP.rotate(x, 3, 100.0)[0]      # angles 3 and 3 / 10
    assert math.isclose(y[0], math.cos(3) - 3 * math.sin(3)) and math.isclose(y[2], 3 * math.cos(3) + math.sin(3))
    assert math.isclose(y[1], 2 * math.cos(0.3) - 4 * math.sin(0.3))
    a, b = np.array([[0.5, -1, 2, 1]]), np.array([[1, 3, -2, 0.25]])   # products depend on the difference alone
    p = OP.rotate(a, 11, 50.0) @ OP.rotate(b, 4, 50.0).T
    assert np.allclose(p, OP.rotate(a, 107, 50.0) @ OP.rotate(b, 100, 50.0).T)


def test_entries_and_new_rows():
    assert OP.entries(5, [3, -1, 9], 2, 9) == [(3, 0), (3, 1)]          # page 9 is outside, page -1 is none
    assert OP.entries(99, [0, 1], 2, 4) == [(0, 0), (0, 1), (1, 0), (1, 1)]
    written, every = OP.append_rows([3, 1, 0], [2, 2, 1], [[5, 6], [7, 8], [1, 1]], 2, 9)
    assert every == [(0, 1), (1, 2), (2, -1), (3, 0), (4, -1)]
    assert written == [(0, 5, 1), (1, 6, 0), (3, 7, 0)]


def test_attention_and_selection():
    o, lse, _, _ = OP.attend([[1.0, 0.0]], [[2.0, 5.0], [2.0, -1.0]], [[1.0, 4.0], [3.0, 0.0]], 0.5)
    assert np.allclose(o, [[2.0, 2.0]]) and np.allclose(lse, 1 + math.log(2))
    o, lse, _, _ = OP.attend(np.ones((2, 4)), np.zeros((0, 4)), np.zeros((0, 4)), 1.0)
    assert not o.any() and np.all(lse == -np.inf)
    s = OP.page_scores([[1.0, -2.0], [0.5, 1.0]], [[[0, 0], [1, 1]], [[-1, -3], [2, 4]]])
    assert list(s) == [1 + 0 + 0.5 + 1, 2 + 6 + 1 + 4]
    assert OP.choose_pages([1.0, 5.0, 5.0, 0.0], [True] * 4, 2, 0, 1) == [1, 3]
    assert OP.choose_pages([1.0, math.nan, 5.0, 0.0], [True, True, False, True], 2, 0, 0) == [0, 3]


def test_logprobs():
    lp, rank, h, ids, top = OP.logprobs([0.0, math.log(2), 0.0, -math.inf], 2, 4)
    assert math.isclose(lp, math.log(0.25)) and rank == 3 and ids == [1, 0, 2, 3]
    assert math.isclose(h, 1.5 * math.log(2)) and top[3] == -math.inf
    assert OP.logprobs([1.0, 1.0], -1, 0)[:2] == (0.0, 0)
    assert all(math.isnan(OP.logprobs(x, 0, 1)[2]) for x in ([-math.inf] * 2, [math.inf, 0], [math.nan, 0]))
