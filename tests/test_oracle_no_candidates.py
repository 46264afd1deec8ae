"""Pins of the oracles where a row allows fewer than k tokens (idx -1, confidence 0): hand-worked values (CPU only)."""

import math

import numpy as np
import pytest

from oracle.accept import accept_sequence, is_consistent, threshold_step
from oracle.brute import consistent_scalar
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


def test_a_step_unmasks_no_position_without_a_token():
    state = np.array([-1, -1, 6, -1])
    conf = np.array([[0, 0], [0.3, 0], [0, 0], [0, 0]], np.float32)
    idx = np.array([[-1, -1], [8, -1], [1, 2], [-1, -1]])
    assert threshold_step(state, conf, idx, 0.9).tolist() == [-1, 8, 6, -1]
    assert threshold_step(state, conf, idx, -1.0).tolist() == [-1, 8, 6, -1]
    # a token of confidence 0 is taken before the positions without one
    assert threshold_step(state, 0 * conf, idx, 0.9).tolist() == [-1, 8, 6, -1]
    idx[1] = -1
    assert threshold_step(state, 0 * conf, idx, 0.9) is None
    for mode in ("exact", "top1", "topk"):
        for check in (is_consistent, consistent_scalar):
            assert not check(state, state, 0 * conf, idx, 0.9, mode)  # a copy is no step


def test_nothing_is_accepted_where_nothing_is_allowed():
    state = np.array([-1, -1])
    none, zero = np.full((2, 2), -1), np.zeros((2, 2), np.float32)
    drafts = np.array([[-1, -1], [5, -1]])
    for tau in (0.9, -1.0):
        for traversal in ("greedy", "longest"):
            r = accept_sequence(drafts, np.array([-1, -1]), state, zero, none, np.stack([zero] * 2), np.stack([none] * 2), tau, "exact", traversal)
            assert r["leaf"] == -1 and r["n_accepted"] == 0 and not r["on_path"].any() and not r["hi"].any()
            assert r["out_tokens"].tolist() == [-1, -1]


@pytest.mark.parametrize("seed", range(30))
def test_consistency_against_sets_of_positions(seed):
    rng = np.random.default_rng(seed)
    L, k, tau = 6, 3, 0.5
    state = np.where(rng.random(L) < 0.7, -1, 50)
    conf = np.sort(rng.random((L, k)))[:, ::-1].astype(np.float32)
    idx = rng.integers(0, 3, (L, k))
    none = np.arange(k) >= rng.integers(0, 3, L)[:, None]
    conf[none], idx[none] = 0, -1
    step = threshold_step(state, conf, idx, tau)
    children = [state] + ([] if step is None else [step]) + [np.where(rng.random(L) < 0.5, idx[:, 0], state) for _ in range(4)]
    for child in children:
        for mode in ("exact", "top1", "topk"):
            assert is_consistent(child, state, conf, idx, tau, mode) == consistent_scalar(child, state, conf, idx, tau, mode)
