"""Prompts written to a paged cache and attended to causally: many row tiles per sequence, each with its own last key, in
ragged batches.  Tolerances as for single blocks: weights of 16 bits, fp32 sums over up to n keys, the output's half step."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import cuda
from oracle.layer import bf16_round

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("T,Hq,Hkv,D,ps,before,n_new", [
    (1500, 7, 1, 128, 16, [0, 40], [1500, 700]),
    (777, 4, 2, 64, 48, [300, 0, 5], [777, 1, 0]),
    (2050, 2, 1, 64, 20, [0], [2050]),
])
def test_a_prompt_attends_to_itself(T, Hq, Hkv, D, ps, before, n_new):
    rng = np.random.default_rng(T)
    B = len(before)
    lens = np.add(before, n_new).astype(np.int32)
    columns = -(-int(lens.max()) // ps)
    pages = B * columns
    table = rng.permutation(pages).reshape(B, columns).astype(np.int32)
    pools = [bf16_round(rng.standard_normal((pages, ps, Hkv, D))) for _ in range(2)]
    q, k, v = (bf16_round(rng.standard_normal((B, T, h, D))) for h in (Hq, Hkv, Hkv))
    up = lambda x: cuda(x.astype(np.float32), BF)  # noqa: E731
    gk, gv, t, new = up(pools[0]), up(pools[1]), cuda(table), cuda(np.array(n_new, np.int32))
    tsp.paged_append(up(k), up(v), gk, gv, t, cuda(np.array(before, np.int32)), n_new=new, rope_theta=0.0)
    _, kp, vp = oracle.paged_append(None, k, v, *pools, table, before, n_new, theta=0)
    assert np.array_equal(f64(gk), kp) and np.array_equal(f64(gv), vp)
    out = f64(tsp.paged_attn(up(q), gk, gv, t, cuda(lens), causal=True, n_new=new))
    assert tsp.device_status() == 0
    for b in range(B):
        assert not out[b, n_new[b]:].any()
        # every tile's first and last rows, some between
        rows = np.unique(np.concatenate([np.arange(0, n_new[b], 16), np.arange(15, n_new[b], 16), rng.integers(0, max(n_new[b], 1), 20),
                                         [n_new[b] - 1]])) if n_new[b] else np.empty(0, int)
        for i in rows:
            n = before[b] + int(i) + 1  # one new token of a sequence that ends with it
            ref, weight = oracle.paged_attention(q[b:b + 1, i:i + 1], kp, vp, table[b:b + 1], [n])
            # scores of up to some 30: their fp32 sums of D products are off by 30 D 2^-24 at most, weights by as much
            tol = (2.0 ** -16 + 2 * n * 2.0 ** -24 + 2 * 30 * D * 2.0 ** -24) * weight + 2.0 ** -8 * np.abs(ref)
            assert (np.abs(out[b, i] - ref[0, 0]) <= tol[0, 0]).all(), (b, i)
