"""Bias lists of many entries: sums in the order of the list, and a cost that goes by its length."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import CONF_ATOL, cuda

pytestmark = pytest.mark.gpu


def call(x, ids, bias, k=8, **more):
    return tsp.confidence_topk_adjusted(x, k, x.shape[0], bias_ids=ids, bias=bias, **more)


def check(x, ids, bias, k=8, **more):
    conf, idx = call(cuda(x), cuda(ids), cuda(bias), k, **{n: cuda(v) for n, v in more.items()})
    rc, ri = oracle.confidence_topk_adjusted(x, k, x.shape[0], bias_ids=ids, bias=bias, **more)
    assert np.array_equal(idx.cpu().numpy(), ri)
    assert np.abs(conf.cpu().numpy() - rc).max() <= CONF_ATOL


@pytest.mark.parametrize("V,NB,most", [(700, 1023, 3), (700, 1025, 8), (5000, 3000, 2), (5000, 4100, 700), (1 << 19, 9000, 6), (4000, 2500, 2500)])
def test_sums_in_the_order_of_the_list(V, NB, most):
    """Tokens named from once to `most` times, anywhere in the list, with biases whose sum depends on the order."""
    rng = np.random.default_rng(V + NB)
    ids = np.empty(0, np.int32)
    while len(ids) < NB:
        ids = np.concatenate([ids, np.full(rng.integers(1, most + 1), rng.integers(0, V), np.int32)])
    ids = rng.permutation(ids[:NB])[None]
    # 2^25 + 1 is 2^25 in fp32: which of the others are lost follows from the order
    bias = rng.choice(np.array([2.0 ** 25, -2.0 ** 25, 1.0, 3.0, 0.25], np.float32), (1, NB))
    x = rng.standard_normal((2, V)).astype(np.float32)
    check(x, ids, bias)
    check(x, ids, bias, history=rng.integers(-1, V, (1, 2000)).astype(np.int32), frequency=np.array([0.5], np.float32))


def test_order_across_and_within_parts_of_a_list():
    """The sum of one token's 2^25, 1 and -2^25 is 0 in this order and 1 in another."""
    big = 2.0 ** 25
    for NB, at, y, want in ((2500, [3, 1100, 2300], [big, 1, -big], 0.0), (2500, [3, 1100, 2300], [big, -big, 1], 1.0),
                            (40, range(10), [big, 1, -big] * 3 + [5], 5.0), (3000, range(0, 3000, 5), [1, big, 1, -big, 1, 0] * 100, 1.0)):
        ids = np.full((1, NB), -1, np.int32)
        bias = np.zeros((1, NB), np.float32)
        ids[0, list(at)], bias[0, list(at)] = 5, y
        x = np.full((1, 64), -40.0, np.float32)
        x[0, 5], x[0, 9] = 0.0, 2.0
        check(x, ids, bias, 3)
        conf, idx = call(cuda(x), cuda(ids), cuda(bias), 2)
        assert abs(float(conf[0, idx[0].tolist().index(5)]) - 1 / (1 + np.exp(2 - want))) <= CONF_ATOL


def best_time(f):
    f()
    times = []
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


def test_a_repeated_token_does_not_slow_the_others_down():
    """16384 ids, all distinct or one of them five times: the same work but for one token's rounds."""
    V, NB = 126464, 16384
    x = torch.randn(2, V, device="cuda")
    ids = torch.randperm(V, device="cuda")[:NB].to(torch.int32)[None].contiguous()
    bias = torch.randn(1, NB, device="cuda")
    distinct = best_time(lambda: call(x, ids, bias))
    ids[0, 1:5] = ids[0, 0]
    assert best_time(lambda: call(x, ids, bias)) < 3 * distinct
