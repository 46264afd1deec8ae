"""Appends in front of tokens that stay (CPU): the oracle by hand, and what the C call refuses."""

import ctypes
import os

import numpy as np
import pytest

from oracle import eight
from paper_2608_27514_amd import _lib
from test_eight_refusals import FAKE, NULL, ODD, SHAPE, ARG, shape


def block(byte, ps=8, H=1, D=64, seed=0):
    """One page of one block with this scale byte."""
    rng = np.random.default_rng(seed)
    values = eight.e4m3(np.clip(100 * rng.standard_normal((2, 1, ps, H, D)), -448, 448))
    return [*values, np.full((1, 1, H), byte), np.full((1, 1, H), byte)]


TABLE = np.array([[0]])


def test_rows_behind_lose_their_values_without_a_length_and_keep_them_with_one():
    before = block(120)
    was = eight.paged_values(before[0], before[2])
    for size, grown in ((2.0 ** -9, 120), (448 * 2.0 ** -3, 124)):  # less than the block has, and more
        x = np.full((1, 2, 1, 64), size)
        _, lost, _ = eight.paged_append8(None, x, x, before, TABLE, [3], theta=0)
        _, kept, _ = eight.paged_append8(None, x, x, before, TABLE, [3], theta=0, lens=[7])
        assert kept[2] == kept[3] == grown
        now = eight.paged_values(kept[0], kept[2])
        stay = [0, 1, 2, 5, 6]
        # a larger scale costs what falls into its subnormals: half a step of 2^-9 of it
        assert (np.abs(now[0, stay] - was[0, stay]) <= 2.0 ** -10 * eight.scale_value(grown) * (grown > 120)).all()
        assert np.array_equal(kept[0][0, 7], before[0][0, 7])  # behind the sequence: bits
        if grown > 120:
            assert not np.array_equal(eight.paged_values(lost[0], lost[2])[0, 5:7], was[0, 5:7])
    # a call at the block's begin: the scale falls without a length, and stays with one
    small = np.full((1, 3, 1, 64), 2.0 ** -9)
    _, lost, _ = eight.paged_append8(None, small, small, before, TABLE, [0], theta=0)
    _, kept, _ = eight.paged_append8(None, small, small, before, TABLE, [0], theta=0, lens=[8])
    assert lost[2] < 120 and kept[2] == 120 and np.array_equal(kept[0][0, 3:], before[0][0, 3:])


@pytest.mark.parametrize("lens", [-5, 0, 4, 5])
def test_a_length_that_ends_with_the_call_keeps_nothing(lens):
    before = block(120)
    x = np.random.default_rng(1).standard_normal((1, 2, 1, 64))
    a = eight.paged_append8(None, x, x, before, TABLE, [3], theta=0)[1]
    b = eight.paged_append8(None, x, x, before, TABLE, [3], theta=0, lens=[lens])[1]
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libtrajspec.so not built")
def test_refusals():
    def call(sh=None, sb=16, theta=1e4, **kw):
        sh = sh or shape()
        a = dict(q=FAKE, qs=8 * 128, k=FAKE, ks=4 * 128, v=FAKE, vs=4 * 128, qo=FAKE, kp=FAKE, vp=FAKE, ksc=FAKE, vsc=FAKE, table=FAKE,
                 start=FAKE, n=None, pos=None, lens=FAKE)
        a.update(kw)
        return _lib.load().traj_paged_append_eight_within(*a.values(), ctypes.byref(sh), sb, theta, None)

    assert call(shape(T=0), k=None) == 0 and call(shape(B=0)) == 0
    assert call(sb=5) == SHAPE and call(shape(Hkv=3)) == SHAPE and call(k=ODD) == SHAPE and call(theta=-1.0) == ARG
    for name in ("k", "v", "kp", "vp", "ksc", "vsc", "table", "start", "q", "qo"):
        assert call(**{name: None}) == NULL, name
    assert _lib.load().traj_paged_append_eight_within(*[FAKE, 8, FAKE, 8, FAKE, 8], *[FAKE] * 10, None, 16, 1.0, None) == NULL
