"""The exact 8-bit products (CPU): their sums against the oracle, what a mistake in one block of k does to them, and which kernels and
ranges of k they reach."""

import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import eight
from paper_2608_27514_amd import _lib
from test_gpu_eight_products import BF, LONG, U8, WIDE, least, operands, product64


def oracle_operands(x, w8, scale):
    K = 64 * w8.shape[0]
    return x.double().numpy(), w8.double().transpose(1, 2).reshape(K, -1).numpy(), scale.view(U8).t().numpy().astype(np.int64)


def to_bf16(y):
    return torch.from_numpy(np.ascontiguousarray(y)).to(BF)


@pytest.mark.parametrize("M,K,N", [(17, 520, 8), (3, 1160, 264), (1, 640, 72)])
def test_the_sums_are_the_oracles(M, K, N):
    x, w8, scale = operands(M, K, N, "cpu")
    xs, values, byte = oracle_operands(x, w8, scale)
    assert np.array_equal(eight.quantize_rows8(xs), xs) and not values[K:].any()
    y, size = eight.linear8(xs, values, byte)
    assert np.array_equal(y, product64(x, w8, scale).numpy())
    assert np.array_equal(y * 8, np.round(y * 8)) and size.max() < 2.0 ** 21


@pytest.mark.parametrize("M,K,N", [(17, 65536, 8), (17, 16512, 8), (1, 65536, 64)])
def test_a_lost_block_or_a_wrong_scale_shows(M, K, N):
    """Each block of 128 of k left out, counted twice (a scale that is twice too large) or with the next block's scale: the
    result differs somewhere.  The bound of the products' other tests would let all of them pass at these lengths."""
    x, w8, scale = operands(M, K, N, "cpu")
    xs, values, byte = oracle_operands(x, w8, scale)
    w = eight.dequantize8(values, byte)
    parts = np.stack([xs[:, 128 * b:128 * b + 128] @ w[128 * b:128 * b + 128] for b in range(byte.shape[0])])
    y = parts.sum(0)
    want = to_bf16(y)
    ref, size = eight.linear8(xs, values, byte)
    assert np.array_equal(y, ref) and size.max() < 2.0 ** 21
    for b in range(byte.shape[0]):
        assert not torch.equal(to_bf16(y - parts[b]), want), b
        assert not torch.equal(to_bf16(y + parts[b]), want), b
        n = (b + 1) % byte.shape[0]
        if (byte[b] != byte[n]).all():
            assert not torch.equal(to_bf16(y + parts[b] * (2.0 ** (byte[n, 0] - byte[b, 0]) - 1)), want), b


@pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libtrajspec.so not built")
def test_kernels_and_ranges_that_are_reached():
    fn = _lib.load().traj_test_gemm_eight_ranges
    fn.restype, fn.argtypes = None, [ctypes.c_int64] * 3 + [ctypes.c_size_t, ctypes.POINTER(ctypes.c_int32)]

    def plan(M, K, N, room):
        out = (ctypes.c_int32 * 3)()
        fn(M, K, N, room, out)
        return tuple(out)

    plans = [plan(*c, least(c[0], c[1])) for c in LONG]
    assert all(ranges == 1 and blocks == -(-c[1] // 128) for (_, ranges, blocks), c in zip(plans, LONG))
    # column scales: a byte per 64 blocks of k, a word per 256
    for longest in (64, 128, 256):
        assert {k for k, _, blocks in plans if blocks > longest and k < 6} == {1, 2, 3, 4, 5}, longest
    assert {k for k, _, _ in plans if k >= 6} == set(range(6, 15))
    wide = {c: plan(*c, _lib.load().traj_linear_eight_workspace_size(*c)) for c in WIDE}
    assert wide[1024, 12288, 4096][1:] == (1, 96) and wide[33, 12288, 4096][0] == 0
