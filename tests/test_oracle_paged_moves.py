"""Pins of the oracle's 8-bit rows, drafts and beams on cases that can be done by hand."""
import math

import numpy as np

from oracle import paged as OP


def test_e4m3_rows():
    assert OP.e4m3([448.0, 1.0, 0.0]) == ([448.0, 1.0, 0.0], 127)
    assert OP.e4m3([449.0, 1.0]) == ([224.0, 0.5], 128)              # 224.5 is nearer to 224 than to 240
    assert OP.e4m3([0.875, -0.0625]) == ([448.0, -32.0], 127 - 9)
    v, b = OP.e4m3([256.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 5 * 2.0 ** -10])
    assert b == 127 and v == [256.0, 16.0, 20.0, 0.0, 2.0 ** -8, 2.0 ** -8]     # halves go to the even one
    v, b = OP.e4m3([math.inf, math.nan, 3.0, -math.inf])
    assert b == 127 - 7 and v[2] == 384.0 and all(math.isnan(x) for x in (v[0], v[1], v[3]))
    assert OP.e4m3([0.0, 0.0]) == ([0.0, 0.0], 10)
    assert OP.e4m3([3.38e38]) == ([240.0], 247)                      # 256 would be 2^128
    rng = np.random.default_rng(0)
    x = rng.standard_normal(512)
    v, b = OP.e4m3(x)
    y = np.asarray(v) * 2.0 ** (b - 127)
    assert np.abs(v).max() > 224 and (np.abs(y - x) <= np.maximum(np.abs(x) / 16, 2.0 ** (b - 127 - 10))).all()


def test_drafts():
    assert OP.visible(7, 3, 0b101, 100) == [0, 1, 2, 3, 4, 6]
    assert OP.visible(7, 3, 0, 100) == [0, 1, 2, 3]
    assert OP.visible(7, 3, 0b110, 6) == [0, 1, 2, 3, 5]
    assert OP.visible(2, 3, 0b110, 100) == [0, 1] and OP.visible(-1, 2, 3, 9) == []
    assert OP.kept_moves(10, 4, [0, 2, 3, -1]) == [(6, 6), (7, 8), (8, 9)]
    assert OP.kept_moves(10, 4, [1, 1, 3]) == [(6, 7)] and OP.kept_moves(10, 4, [4]) == []


def test_beams():
    new, copies = OP.reordered([[1, 2, 3], [1, 5, 6], [7, 8, 9], [7, 11, 12]], [5, 0, 4, 4], [1, 0, -1, 0], 2, 4)
    assert new == [[1, 2, 3], [1, 5, 6], [7, 8, 9], [7, 11, 12]] and copies == [(2, 5, 1), (5, 2, 1)]
    new, copies = OP.reordered([[1, 2, 3], [4, 5, 6]], [9, 9], [1, 1], 2, 4)
    assert new == [[4, 5, 3], [4, 5, 6]] and copies == [(3, 6, 1)]
    x = np.log([[1.0, 2.0, 1.0], [8.0, 1.0, 1.0]])
    got = OP.beam_select(x, [-1.0, -1.0], None, 0, 3)
    assert [g[:2] for g in got] == [(1, 0), (0, 1), (0, 0)] and math.isclose(got[0][2], -1 + math.log(0.8))
    got = OP.beam_select(x, [-1.0, -2.0], [0, 1], 7, 6)
    assert [g[:2] for g in got] == [(0, 1), (1, 7), (0, 0), (0, 2), (-1, -1), (-1, -1)]
    assert OP.beam_select(x, [-math.inf, math.nan], None, 0, 1) == [(-1, -1, -math.inf)]
