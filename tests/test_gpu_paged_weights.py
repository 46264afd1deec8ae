"""The softmax weights of the paged attention reach the product with V to 16 bits, whatever the number of rows.

Values +v and -v under weights of 1 and exp(-2^-9) nearly cancel, so that the output's own rounding does not hide the
weights': exp(-2^-9) = 0.998049 lies in the middle of two bf16 values, and a weight of 8 bits moves the output by 2^-10
of the sum of w |v|.  With weights in two bf16 parts each is off by half a step of half a step, 2^-16 of itself; the
scores are one product each, their exponentials within 2^-20; fp32 sums of n weights and of n products by n 2^-24 each.
So |err| <= (2^-16 + 2^-20 + 2 n 2^-24) sum w |v| + 2^-8 |out|, the last for the output's rounding."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import cuda
from oracle.layer import bf16_round

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("lens", [[200, 37], [3000, 50]])
@pytest.mark.parametrize("ps", [16, 5])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 2), (13, 4, 2), (32, 4, 2), (64, 4, 2), (70, 8, 2)])  # a kernel each
def test_weights_to_16_bits(T, Hq, Hkv, D, ps, lens):
    rng = np.random.default_rng(T + D + ps)
    B = len(lens)
    columns = -(-max(lens) // ps)
    pages = B * columns
    table = rng.permutation(pages).reshape(B, columns).astype(np.int32)
    kp, vp = np.zeros((pages, ps, Hkv, D)), np.zeros((pages, ps, Hkv, D))
    odd = rng.permuted(np.arange(pages * ps * Hkv) % 2).reshape(pages, ps, Hkv)
    scale = D ** -0.5 if D == 64 else 0.125
    kp[..., 0] = -odd / 64.0  # scores 0 and -1 / 512
    vp[:] = np.where(odd[..., None] == 1, -1.0, 1.0) * bf16_round(0.5 + rng.random((Hkv, D)))
    q = np.zeros((B, T, Hq, D))
    q[..., 0] = 1.0
    ref, weight = oracle.paged_attention(q, kp, vp, table, lens, scale=scale)
    up = lambda x: cuda(x.astype(np.float32), BF)  # noqa: E731
    out = tsp.paged_attn(up(q), up(kp), up(vp), cuda(table), cuda(np.array(lens, np.int32)), scale=scale)
    err = np.abs(out.float().cpu().numpy().astype(np.float64) - ref)
    n = np.array(lens)[:, None, None, None]
    assert (err <= (2.0 ** -16 + 2.0 ** -20 + 2 * n * 2.0 ** -24) * weight + 2.0 ** -8 * np.abs(ref)).all(), err.max()
