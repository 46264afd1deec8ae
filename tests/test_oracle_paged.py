"""Pins of the paged-cache and adjusted-logits oracles (CPU): library routines, invariants, hand-worked values."""

import numpy as np
import pytest
import torch

import oracle


def pool(rng, B, columns, ps, Hkv, D):
    pages = B * columns + 2
    return rng.permutation(pages)[:B * columns].reshape(B, columns), rng.standard_normal((pages, ps, Hkv, D)), rng.standard_normal((pages, ps, Hkv, D))


@pytest.mark.parametrize("causal", [False, True])
def test_attention_is_library_attention_over_the_gathered_keys(causal):
    rng = np.random.default_rng(1)
    B, T, Hq, Hkv, D, ps = 2, 3, 6, 2, 64, 5
    table, kp, vp = pool(rng, B, 4, ps, Hkv, D)
    q = rng.standard_normal((B, T, Hq, D))
    lens = [17, 9]
    out, weight = oracle.paged_attention(q, kp, vp, table, lens, causal)
    for b, n in enumerate(lens):
        k = torch.from_numpy(kp[table[b]].reshape(-1, Hkv, D)[:n]).permute(1, 0, 2).repeat_interleave(3, 0)
        v = torch.from_numpy(vp[table[b]].reshape(-1, Hkv, D)[:n]).permute(1, 0, 2).repeat_interleave(3, 0)
        mask = torch.ones(T, n, dtype=torch.bool).tril(n - T) if causal else None
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[b]).permute(1, 0, 2), k, v, attn_mask=mask)
        assert np.abs(out[b] - want.permute(1, 0, 2).numpy()).max() < 1e-12
    assert (weight >= np.abs(out) - 1e-12).all()


def test_attention_ignores_what_is_not_visible():
    rng = np.random.default_rng(2)
    table, kp, vp = pool(rng, 1, 3, 4, 1, 64)
    q = rng.standard_normal((1, 2, 2, 64))
    a, _ = oracle.paged_attention(q, kp, vp, table, [6])
    kp[table[0, 1], 2:], vp[table[0, 1], 2:], kp[table[0, 2]] = np.nan, np.inf, 3.0
    b, _ = oracle.paged_attention(q, kp, vp, table, [6])
    assert np.array_equal(a, b)
    table[0, 0] = -1  # a page that is none: its keys are gone
    c, _ = oracle.paged_attention(q, kp, vp, table, [6])
    d, _ = oracle.paged_attention(q, kp, vp, table[:, 1:], [2])
    assert np.array_equal(c, d)
    assert not oracle.paged_attention(q, kp, vp, table, [0])[0].any()
    causal, _ = oracle.paged_attention(q, kp, vp, table[:, 1:], [1], causal=True)
    assert not causal[0, 0].any() and np.array_equal(causal[0, 1, 0], vp[table[0, 1], 0, 0])


def test_rotation_keeps_norms_and_relative_scores():
    rng = np.random.default_rng(3)
    x, y = rng.standard_normal((2, 4, 1, 64))
    p = np.array([0, 5, 100, 7000])
    r = oracle.rotate(x, p, 10000.0)
    assert np.array_equal(r[0], x[0]) and np.allclose((r ** 2).sum(-1), (x ** 2).sum(-1))
    s = (oracle.rotate(x, p, 10000.0) * oracle.rotate(y, p + 3, 10000.0)).sum(-1)
    t = (oracle.rotate(x, p + 40, 10000.0) * oracle.rotate(y, p + 43, 10000.0)).sum(-1)
    assert np.allclose(s, t)
    unit = np.zeros((1, 1, 64))
    unit[..., 0] = 1  # the first pair turns by the position itself
    turned = oracle.rotate(unit, np.array([2]), 10000.0)
    assert np.allclose(turned[0, 0, [0, 32]], [np.cos(2), np.sin(2)])


def test_append_puts_tokens_in_their_rows():
    rng = np.random.default_rng(4)
    B, T, H, D, ps = 2, 3, 1, 64, 2
    table = np.array([[4, 1, 0], [2, 3, 5]])
    k, v, q = rng.standard_normal((3, B, T, H, D))
    kp, vp = np.zeros((6, ps, H, D)), np.zeros((6, ps, H, D))
    out, k2, v2 = oracle.paged_append(q, k, v, kp, vp, table, [1, 4], n_new=[3, 1], pos0=[10, 20])
    at = [(4, 1, 0, 0), (1, 0, 0, 1), (1, 1, 0, 2), (5, 0, 1, 0)]  # page, row, sequence, token
    for page, row, b, t in at:
        assert np.array_equal(v2[page, row], v[b, t])
        assert np.array_equal(k2[page, row], oracle.rotate(k[b, t], 10 * (b + 1) + t, 500000.0))
        v2[page, row] = k2[page, row] = 0
    assert not v2.any() and not k2.any() and not kp.any()
    assert not out[1, 1:].any() and np.array_equal(out[0, 2], oracle.rotate(q[0, 2], 12, 500000.0))


def test_adjusted_values_by_hand():
    x = np.array([[2.0, -2.0, 1.0, 0.5, 3.0, 4.0]], np.float32)
    how = dict(history=np.array([[0, 1, 0, -1, 9, 2]]), history_len=[5], repetition=[4.0], frequency=[0.25], presence=[0.5],
               bias_ids=np.array([[2, 2, 1, -1]]), bias=np.array([[1.0, 2.0, 8.0, 100.0]], np.float32),
               mask=np.array([[0b011111]], np.uint32), mask_index=[0])
    y = oracle.adjust_logits(x, 1, **how)
    # 2 / 4 - (2 * 0.25 + 0.5);  -2 * 4 + 8 - (0.25 + 0.5);  1 + 3;  unchanged;  unchanged;  forbidden
    assert y.tolist() == [[-0.5, -0.75, 4.0, 0.5, 3.0, -np.inf]]
    conf, idx = oracle.confidence_topk_adjusted(x, 6, 1, **how)
    assert idx.tolist() == [[2, 4, 3, 0, 1, -1]] and conf[0, 5] == 0 and abs(conf.sum() - 1) < 1e-12


def test_adjusting_nothing_is_the_plain_pass():
    rng = np.random.default_rng(5)
    x = np.round(rng.standard_normal((5, 200)), 1).astype(np.float32)  # many ties
    conf, idx = oracle.confidence_topk_adjusted(x, 8, 2)
    want = oracle.confidence_topk(x, 8)
    assert np.array_equal(idx, want[1]) and np.allclose(conf, want[0], rtol=1e-12)


def test_adjusted_values_against_the_formula_in_64_bits():
    rng = np.random.default_rng(6)
    n, per, V, H = 3, 2, 50, 30
    x = rng.standard_normal((n * per, V)).astype(np.float32)
    h = rng.integers(-1, V + 1, (n, H))
    r, f, p = rng.uniform(0.5, 2, n), rng.uniform(-1, 1, n), rng.uniform(-1, 1, n)
    ids, bias = rng.integers(0, V, (n, 5)), rng.standard_normal((n, 5)).astype(np.float32)
    f32 = lambda a: a.astype(np.float32)  # noqa: E731
    got = oracle.adjust_logits(x, per, history=h, repetition=f32(r), frequency=f32(f), presence=f32(p), bias_ids=ids, bias=bias)
    for row in range(n * per):
        q = row // per
        c = np.array([(h[q] == v).sum() for v in range(V)])
        y = np.where(c > 0, np.where(x[row] > 0, x[row] / r[q], x[row] * r[q]) - f[q] * c - p[q], x[row])
        y = y + np.array([bias[q][ids[q] == v].sum() for v in range(V)])
        assert np.abs(got[row] - y).max() < 2.0 ** -20  # a handful of fp32 roundings of values below 16
    assert np.array_equal(oracle.adjust_logits(x, per, mask=np.zeros((1, 2), np.uint32), mask_index=[-1, 0, 1, -2, -1, -1])[:, 0] == -np.inf,
                          [False, True, True, True, False, False])
