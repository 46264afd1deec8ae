"""Sizes of the serving calls that 32 bits do not hold (CPU only)."""

import ctypes
import os

import pytest

from paper_2608_27514_amd import _lib

BIG = 2 ** 32 + 1  # 1 in 32 bits


def test_the_binding_refuses_sizes_past_32_bits():
    with pytest.raises(ValueError, match="rows_per_seq"):  # as 1, every row would have lists of its own
        _lib._logit_adjust(0, 8, 100, BIG, *[None] * 9)
    assert _lib._logit_adjust(0, 8, 100, 2 ** 31 - 1, *[None] * 9).rows_per_seq == 2 ** 31 - 1
    good = dict(B=1, T=1, Hq=4, pages=(4, 16, 2, 64), strides=(2048, 128, 64, 1), table=(1, 4), table_strides=(4, 1))
    _lib._paged_struct(*good.values())
    for bad in (dict(T=BIG), dict(Hq=BIG), dict(pages=(BIG, 16, 2, 64)), dict(pages=(4, BIG, 2, 64)), dict(pages=(4, 16, BIG, 64)),
                dict(pages=(4, 16, 2, BIG)), dict(table=(1, BIG)), dict(B=BIG, table=(BIG, 4))):
        with pytest.raises(ValueError, match="2\\^31"):
            _lib._paged_struct(*{**good, **bad}.values())


@pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libtrajspec.so not built")
def test_workspace_sizes_of_lists_past_32_bits():
    for bad in (dict(k=BIG), dict(per=BIG), dict(H=BIG), dict(NB=BIG)):
        with pytest.raises(ValueError, match="2\\^31"):
            _lib._adjust_workspace(*{**dict(rows=8, vocab=100, row_stride=100, dtype=0, k=3, per=1, H=4, NB=0), **bad}.values())


@pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libtrajspec.so not built")
def test_head_counts_whose_products_pass_64_bits():
    """B T Hq = 2^65 would count as 0 rows, and a workspace of some arbitrary size would be reported for them."""
    lib = _lib.load()
    for heads in (1 << 30, 1 << 17, 65537):
        for Hkv in (1, heads):
            sh = _lib.PagedShape(2048, 1 << 13 if Hkv == 1 else 1 << 24, heads, Hkv, 128, 10, 16, 4096, 4096, 16 * 512, 512, 128)
            assert lib.traj_paged_attn_workspace_size(ctypes.byref(sh)) == 0
            assert lib.traj_paged_attn(*[0x1000] * 7, ctypes.byref(sh), 0.0, 0, None, 0, None) == 2  # TRAJ_E_SHAPE; nothing is read
            assert lib.traj_paged_append(*[0x1000, 1 << 38] * 3, *[0x1000] * 5, None, None, ctypes.byref(sh), 1e4, None) == 2
