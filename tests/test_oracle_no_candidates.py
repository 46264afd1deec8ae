"""Pins of the oracles where a row allows fewer than k tokens (idx -1, confidence 0): hand-worked values (CPU only)."""

import math

import numpy as np
import pytest

from oracle.tree import build_tree, build_tree_batch

NONE = [-1, -1, -1]


def tree(state, conf, idx, *shape, **kw):
    t, p, s = build_tree(np.array(state), np.array(conf, np.float32), np.array(idx), 0.5, *shape, **kw)
    return t.tolist(), p.tolist(), s.tolist()


def test_a_slot_without_a_token_makes_no_child():
    # position 0 has one allowed token, position 1 two, position 2 none, position 3 is committed
    conf = [[0.4, 0, 0], [0.5, 0.3, 0], [0, 0, 0], [0.9, 0, 0]]
    idx = [[7, -1, -1], [8, 9, -1], NONE, [1, 2, 3]]
    t, p, s = tree([-1, -1, -1, 5], conf, idx, 3, 3, 3, True, branch_deep=3)
    # level 1 at position 1: two children; level 2 at position 0: one each; no level 3
    assert t == [[-1, 8, -1, 5], [-1, 9, -1, 5], [7, 8, -1, 5], [7, 9, -1, 5]]
    assert p == [-1, -1, 0, 1]
    c = np.float32([0.5, 0.3, 0.4]).astype(float)
    assert np.allclose(s, [math.log(c[0]), math.log(c[1]), math.log(c[0]) + math.log(c[2]), math.log(c[1]) + math.log(c[2])])


def test_positions_without_a_token_stay_masked():
    conf = [[0.9, 0, 0], [0, 0, 0]]
    t, p, s = tree([-1, -1], conf, [[4, -1, -1], NONE], 2, 2, 2)
    assert (t, p, s) == ([[4, -1]], [-1], [0.0])  # the root alone
    assert tree([-1, -1], [[0, 0, 0], [0, 0, 0]], [NONE, NONE], 2, 2, 2) == ([], [], [])
    # a threshold below 0 does not make them certain
    assert build_tree(np.array([-1, -1]), np.zeros((2, 3)), np.array([NONE, NONE]), -1.0, 2, 2, 2)[1].size == 0


def test_a_token_of_confidence_0_is_still_a_candidate():
    t, p, s = tree([-1], [[0.4, 0, 0]], [[4, 5, -1]], 3, 1, 3)
    assert t == [[4], [5]] and s[1] == -math.inf


def test_batch_of_nothing():
    t, p, n, s = build_tree_batch(np.array([[-1, 3]]), None, None, None, np.zeros((1, 2, 3)), np.full((1, 2, 3), -1), 0.5, 2, 2, 2, False, 4)
    assert n.tolist() == [0] and t.tolist() == [[[-1, 3]] * 4] and (p == -1).all() and (s == -np.inf).all()
