"""Sizes of the serving calls that 32 bits do not hold (CPU only)."""

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
