"""Prompts written to an 8-bit cache and attended to: many row tiles per sequence, each with its own last key, in ragged batches,
whole and split.  Keys and values enter exactly; scores of up to some 30 are fp32 sums of D products, off by 30 D 2^-24 at
most, and weights by as much and by their cut to 16 bits (2^-16); fp32 sums over up to n keys; the output's half step."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from oracle import eight
from oracle.layer import bf16_round
from test_gpu_eight import E4, bf, bytes_of, f64, heads_first, i32, make_pools, make_table, on_gpu

pytestmark = pytest.mark.gpu

CASES = [
    # T, Hq, Hkv, D, page_size, scale block, cached before, n_new
    (1500, 7, 1, 128, 16, 16, [0, 40], [1500, 700]),          # 83 row tiles
    (777, 4, 2, 64, 48, 24, [300, 0, 5], [777, 1, 0]),
    (2050, 2, 1, 64, 20, 4, [0], [2050]),
    (300, 8, 2, 128, 32, 32, [0, 100, 513], [300, 299, 17]),  # ten tiles that share the keys
    (600, 4, 1, 128, 64, 64, [2100], [600]),                  # behind a long cached part: split
    (333, 16, 4, 64, 5, 5, [0, 77], [333, 200]),              # heads in pairs, pages that end inside every tile
    (130, 1, 1, 128, 24, 8, [0, 0, 900], [130, 129, 2]),
    (1030, 3, 3, 64, 16, 1, [7], [1029]),
]


def rows_to_check(rng, n):
    """Every tile's first and last rows, some between."""
    return np.unique(np.concatenate([np.arange(0, n, 16), np.arange(15, n, 16), rng.integers(0, max(n, 1), 20), [n - 1]])) if n else np.empty(0, int)


def tolerance(n, D, weight, ref):
    return (2.0 ** -16 + 2 * n * 2.0 ** -24 + 2 * 30 * D * 2.0 ** -24) * weight + 2.0 ** -8 * np.abs(ref)


@pytest.mark.parametrize("T,Hq,Hkv,D,ps,sb,before,n_new", CASES)
def test_a_prompt_attends_to_itself(T, Hq, Hkv, D, ps, sb, before, n_new):
    rng = np.random.default_rng(T)
    B = len(before)
    lens = np.add(before, n_new).astype(np.int32)
    table, pages = make_table(rng, B, -(-int(lens.max()) // ps))
    pools = make_pools(rng, pages, ps, sb, Hkv, D)
    q, k, v = (bf16_round(rng.standard_normal((B, T, h, D))) for h in (Hq, Hkv, Hkv))
    got, t, new = on_gpu(pools, heads_first if T % 2 else lambda x: x), i32(table), i32(n_new)
    tsp.paged_append8(bf(k), bf(v), *got, t, i32(before), n_new=new, rope_theta=0.0)
    _, pools, _ = eight.paged_append8(None, k, v, pools, table, before, n_new, theta=0)
    assert all(np.array_equal(f64(x) if x.dtype == E4 else bytes_of(x), want) for x, want in zip(got, pools))
    kp, vp = (eight.paged_values(pools[i], pools[2 + i]) for i in (0, 1))
    padded = bf(q)
    for b in range(B):
        padded[b, n_new[b]:] = float("nan")
    causal = tsp.paged_attn8(padded, *got, t, i32(lens), causal=True, n_new=new)
    full = tsp.paged_attn8(padded, *got, t, i32(lens), n_new=new)
    assert tsp.device_status() == 0
    assert torch.equal(tsp.paged_attn8(padded, *got, t, i32(lens), causal=True, n_new=new), causal)
    for b in range(B):
        assert not causal[b, n_new[b]:].any() and not full[b, n_new[b]:].any()
        rows = rows_to_check(rng, n_new[b])
        for out, upto in ((f64(causal[b]), True), (f64(full[b]), False)):
            for i in rows[:: 1 if upto else 7]:
                n = before[b] + int(i) + 1 if upto else int(lens[b])  # one new token of a sequence that ends with it
                ref, weight = oracle.paged_attention(q[b:b + 1, i:i + 1], kp, vp, table[b:b + 1], [n])
                assert (np.abs(out[i] - ref[0, 0]) <= tolerance(n, D, weight, ref)[0, 0]).all(), (b, i, upto)


def test_a_prompt_in_parts_as_at_once():
    """A prompt appended and attended to in parts that begin and end inside scale blocks: the cache's scales are the whole
    prompt's where a block grows to them, and each part's attention is that over the cache it left."""
    rng = np.random.default_rng(9)
    T, H, D, ps, sb = 700, 2, 64, 32, 16
    table, pages = make_table(rng, 1, -(-T // ps))
    pools = make_pools(rng, pages, ps, sb, H, D)
    q, k, v = (bf16_round(rng.standard_normal((1, T, h, D))) for h in (4, H, H))
    got, t = on_gpu(pools), i32(table)
    for a, e in ((0, 250), (250, 251), (251, 600), (600, 700)):
        tsp.paged_append8(bf(k[:, a:e]), bf(v[:, a:e]), *got, t, i32([a]), rope_theta=0.0)
        _, pools, _ = eight.paged_append8(None, k[:, a:e], v[:, a:e], pools, table, [a], theta=0)
        assert all(np.array_equal(f64(x) if x.dtype == E4 else bytes_of(x), want) for x, want in zip(got, pools))
        kp, vp = (eight.paged_values(pools[i], pools[2 + i]) for i in (0, 1))
        out = f64(tsp.paged_attn8(bf(q[:, a:e]), *got, t, i32([e]), causal=True))
        assert tsp.device_status() == 0
        for i in rows_to_check(rng, e - a):
            ref, weight = oracle.paged_attention(q[:, a + i:a + i + 1], kp, vp, table, [a + int(i) + 1])
            assert (np.abs(out[0, i] - ref[0, 0]) <= tolerance(a + i + 1, D, weight, ref)[0, 0]).all(), (a, i)
