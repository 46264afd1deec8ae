"""Pins of the 8-bit oracle (CPU): library conversions, values by hand, invariants."""

import numpy as np
import torch

import oracle
from oracle import eight


def test_rounding_is_the_library_types():
    """Every e4m3 value, the midpoints between neighbours and values beside them, against torch's conversion."""
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = (codes[1:] + codes[:-1]) / 2
    x = np.concatenate([codes, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(eight.e4m3(x), want)
    assert np.isnan(eight.e4m3([np.nan, np.inf, -np.inf])).all()


def test_scales_by_hand():
    for amax, e in ((448.0, 0), (448.5, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7578125, -7), (0.0, -100), (2.0 ** -120, -100), (3.0e38, 120)):
        assert eight.scale_byte(amax) == 127 + e, amax
    x = np.array([1.0, -3.0, np.inf, np.nan])
    assert eight.scale_byte(eight.magnitude(x).max()) == eight.scale_byte(3.0)
    rng = np.random.default_rng(0)
    a = np.exp(rng.uniform(-60, 80, 1000))
    s = eight.scale_value(eight.scale_byte(a))
    assert (a <= 448 * s).all() and (a > 224 * s).all()


def test_weights_are_off_by_half_a_step():
    rng = np.random.default_rng(1)
    w = rng.standard_normal((200, 136)) * np.exp(rng.standard_normal((200, 1)))
    values, byte = eight.quantize8(w)
    assert values.shape == (256, 136) and byte.shape == (2, 2) and not values[200:].any()
    back, s = eight.dequantize8(values, byte)[:200], eight.scale_value(byte).repeat(128, 0).repeat(128, 1)[:200, :136]
    assert (np.abs(back - w) <= 2.0 ** -4 * np.abs(w) + 2.0 ** -10 * s).all()
    x = rng.standard_normal((3, 200))
    q = eight.quantize_rows8(x)
    y, size = eight.linear8(x, values, byte)
    assert np.allclose(y, q @ back, rtol=1e-12, atol=0) and (size >= np.abs(y)).all()
    assert np.array_equal(eight.quantize_rows8(q), q)  # what has been rounded stays
    bad = x.copy()
    bad[1, 5] = np.inf
    assert np.isnan(eight.linear8(bad, values, byte)[0][1]).all() and np.array_equal(eight.linear8(bad, values, byte)[0][[0, 2]], y[[0, 2]])


def pools(rng, pages, ps, sb, H, D):
    byte = rng.integers(118, 124, (2, pages, ps // sb, H))
    return [*eight.e4m3(100 * rng.standard_normal((2, pages, ps, H, D))), *byte]


def test_append_of_whole_blocks_forgets_what_was_there():
    rng = np.random.default_rng(2)
    B, T, H, D, ps, sb = 2, 8, 2, 64, 8, 4
    table = np.array([[3, 0], [1, 2]])
    k, v = rng.standard_normal((2, B, T, H, D))
    a = eight.paged_append8(None, k, v, pools(rng, 4, ps, sb, H, D), table, [0, 8], theta=0)[1]
    b = eight.paged_append8(None, k, v, pools(rng, 4, ps, sb, H, D), table, [0, 8], theta=0)[1]
    for page, row in ((3, 0), (2, 1)):
        for x, y, want in zip(a[:2], b[:2], (k, v)):
            assert np.array_equal(x[page], y[page])
        for x, y, want in ((a[0], a[2], k), (a[1], a[3], v)):
            got = eight.paged_values(x[page:page + 1], y[page:page + 1])[0]
            s = eight.scale_value(y[page]).repeat(sb, 0)[..., None]
            assert (np.abs(got - want[row]) <= 2.0 ** -4 * np.abs(want[row]) + 2.0 ** -10 * s).all()


def test_append_within_a_block_keeps_its_rows_and_never_shrinks_its_scale():
    rng = np.random.default_rng(3)
    H, D, ps = 1, 64, 8
    table = np.array([[0]])
    start = pools(rng, 1, ps, ps, H, D)
    start[2][:] = start[3][:] = 120
    small = np.full((1, 2, H, D), 2.0 ** -9)
    _, p, exact = eight.paged_append8(None, small, small, start, table, [3], theta=0)
    assert p[2] == 120 and np.array_equal(p[0][0, :3], start[0][0, :3]) and np.array_equal(p[0][0, 5:], start[0][0, 5:])
    assert np.array_equal(p[0][0, 3:5], eight.e4m3(small[0] * 2.0 ** 7)) and np.isnan(exact[0][0, :3]).all()
    large = np.full((1, 1, H, D), 448 * 2.0 ** -3)
    _, p, _ = eight.paged_append8(None, large, small, start, table, [3], theta=0)
    assert p[2] == 124 and p[3] == 120
    assert np.array_equal(p[0][0, :3], eight.e4m3(start[0][0, :3] / 16)) and (p[0][0, 3] == 448).all()
    assert np.array_equal(p[0][0, 4:], start[0][0, 4:]) and np.array_equal(p[1][0, :3], start[1][0, :3])
    # values that stay above the subnormals keep what they stand for
    big = np.abs(start[0][0, :3]) >= 16 * 2.0 ** -6
    assert np.array_equal(eight.paged_values(p[0], p[2])[0, :3][big], eight.paged_values(start[0], start[2])[0, :3][big])


def test_append_token_by_token_ends_near_the_block_at_once():
    """A block filled by single tokens: every value within a step of the block's largest scale."""
    rng = np.random.default_rng(4)
    T, H, D, ps = 16, 2, 64, 16
    k, v = rng.standard_normal((2, 1, T, H, D)) * np.exp(rng.standard_normal((1, T, 1, 1)))
    table = np.array([[1]])
    p = pools(rng, 2, ps, ps, H, D)
    whole = eight.paged_append8(None, k, v, p, table, [0])[1]
    for t in range(T):
        p = eight.paged_append8(None, k[:, t:t + 1], v[:, t:t + 1], p, table, [t])[1]
    assert np.array_equal(p[2][1], whole[2][1]) and np.array_equal(p[3][1], whole[3][1])
    a, b = (eight.paged_values(x[0], x[2])[1] for x in (p, whole))
    s = eight.scale_value(whole[2][1])[..., None]
    assert (np.abs(a - b) <= 2.0 ** -9 * s).all()
    assert np.array_equal(p[0][0], p[0][0]) and oracle.paged_attention(np.ones((1, 1, H, D)), a[None], a[None], np.array([[0]]), [T])[0].shape == (1, 1, H, D)


def test_append_skips_what_has_no_place():
    rng = np.random.default_rng(5)
    H, D, ps, sb = 1, 64, 4, 2
    k = rng.standard_normal((3, 5, H, D))
    before = pools(rng, 4, ps, sb, H, D)
    table = np.array([[0, 9], [-1, 1], [2, 3]])
    _, p, exact = eight.paged_append8(None, k, k, before, table, [2, 2, -3], n_new=[5, 3, 9], theta=0)
    written = ~np.isnan(exact[0]).any((2, 3))
    assert written.tolist() == [[False, False, True, True], [True, False, False, False], [True, True, False, False], [False] * 4]
    assert np.array_equal(p[0][~written], before[0][~written])
