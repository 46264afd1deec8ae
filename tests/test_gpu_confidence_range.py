"""Confidences of logits over their type's whole finite range: masked by its lowest value, wholly or in part, huge ones, and
ones whose product with log2(e) overflows.  Against the oracle, for every launch shape of the pass."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import CONF_ATOL

pytestmark = pytest.mark.gpu


def rows_of(rng, R, V, dtype):
    """Rows of each kind in turn, as a tensor of the type."""
    big = float(torch.finfo(dtype).max)
    x = rng.standard_normal((R, V)).astype(np.float32)
    for r in range(R):
        kind = r % 10
        if kind == 0:
            x[r, rng.random(V) < 0.5] = -big
        elif kind == 1:
            x[r, :-(-V // 2)] = -big  # a lane's first vectors hold nothing else
        elif kind == 2:
            x[r] = -big
            x[r, rng.integers(V)] = 1.0
        elif kind == 3:
            x[r] = -big
        elif kind == 4:
            x[r] = -big
            x[r, ::2] = -np.inf
        elif kind == 5:
            x[r, V // 3] = big
        elif kind == 6:
            x[r] = big
        elif kind == 7:
            x[r] = -1e30 * rng.integers(1, 300, V)
        elif kind == 8:
            x[r, :-(-V // 2)] = (-1e10, -1e9, -1e30)[r // 10 % 3]
        else:
            x[r, : V - 1] = -np.inf
            x[r, V - 1] = -3e38
    return torch.from_numpy(x).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,V", [(10, 50257), (1, 126464), (40, 20000), (300, 5003), (700, 1237), (90, 300), (4600, 257), (18, 8)])
def test_the_whole_finite_range(R, V, dtype):
    x = rows_of(np.random.default_rng(R), R, V, dtype)
    rc, ri = oracle.confidence_topk(x.float().numpy(), 4)
    g = x.cuda()
    calls = [lambda: tsp.confidence_topk(g, 4), lambda: tsp.confidence_topk_noalloc(g, 4)]
    if R < 700:
        none = torch.zeros(0, dtype=torch.uint8, device="cuda")
        calls.append(lambda: tsp.confidence_topk(g, 4, workspace=none))  # rows are not split
    for call in calls:
        conf, idx = call()
        assert np.array_equal(idx.cpu().numpy(), ri)
        assert np.abs(conf.cpu().numpy() - rc).max() <= CONF_ATOL
