"""Lengths that no sequence can have are reported and clamped wherever they stand in the batch, in split and unsplit calls."""

import ctypes

import numpy as np
import pytest
import torch

import paper_2608_27514_amd as tsp
from helpers import cuda
from paper_2608_27514_amd import _lib

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def pool(B, columns, ps=16, Hkv=2, D=64):
    g = torch.Generator(device="cuda")
    g.manual_seed(columns)
    kp, vp = (torch.randn(B * columns, ps, Hkv, D, generator=g, device="cuda").to(BF) for _ in range(2))
    q = torch.randn(B, 1, 2 * Hkv, D, generator=g, device="cuda").to(BF)
    return q, kp, vp, torch.arange(B * columns, device="cuda", dtype=torch.int32).view(B, columns)


def unsplit(q, kp, vp, table, lens):
    """A call with no workspace."""
    sh = _lib._paged_struct(*_lib._paged_sizes(*q.shape[:3], kp, vp, table, 0))[0]
    out = torch.empty_like(q)
    ptr = [x.data_ptr() for x in (q, kp, vp, table, lens)] + [None, out.data_ptr()]
    assert tsp.load().traj_paged_attn(*ptr, ctypes.byref(sh), 0.0, 0, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    return out


CALLS = [
    # sequences, table columns, call: a cache that is never split, a split one, one without a workspace, too many sequences
    (4, 3, tsp.paged_attn),
    (4, 60, tsp.paged_attn),
    (4, 60, unsplit),
    (2100, 20, tsp.paged_attn),
]


@pytest.mark.parametrize("B,columns,call", CALLS)
@pytest.mark.parametrize("bad", [-1, 1 << 30])
@pytest.mark.parametrize("at", [0, 1, -1])
def test_a_bad_length_anywhere_is_reported(B, columns, call, bad, at):
    q, kp, vp, table = pool(B, columns)
    lens = np.full(B, 7, np.int32)
    tsp.device_status()
    call(q, kp, vp, table, cuda(lens))
    assert tsp.device_status() == 0
    lens[at] = bad
    out = call(q, kp, vp, table, cuda(lens))
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH
    lens[at] = 0 if bad < 0 else columns * 16
    assert torch.equal(out, call(q, kp, vp, table, cuda(lens)))
    assert tsp.device_status() == 0
