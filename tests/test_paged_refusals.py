"""What the paged-cache and adjusted-logits calls refuse, before anything reaches the device (CPU only)."""

import ctypes
import math
import os

import pytest
import torch

import paper_2608_27514_amd as tsp
from paper_2608_27514_amd import _lib

pytestmark = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libtrajspec.so not built")
FAKE, ODD = 0x1000, 0x1008  # never dereferenced
NULL, SHAPE, DTYPE, UNSUPPORTED, WORKSPACE, ARG = 1, 2, 3, 4, 5, 7


def shape(**kw):
    d = dict(B=2, T=3, Hq=8, Hkv=4, D=128, num_pages=10, page_size=16, max_pages=4, table_stride=4, page_stride=16 * 512, token_stride=512,
             head_stride=128)
    return _lib.PagedShape(**{**d, **kw})


BAD_SHAPES = [dict(B=-1), dict(B=65536), dict(T=-1), dict(Hq=0), dict(Hkv=0), dict(Hkv=3), dict(num_pages=0), dict(page_size=0), dict(max_pages=0),
              dict(max_pages=1 << 20, page_size=1 << 11, table_stride=1 << 20), dict(T=(1 << 24) + 1),
              dict(max_pages=(1 << 31) - 4095, page_size=1, table_stride=1 << 31), dict(table_stride=3), dict(page_stride=12), dict(token_stride=0),
              dict(head_stride=-8), dict(T=1 << 30)]


def append(sh=None, theta=1e4, **kw):
    sh = sh or shape()
    a = dict(q=FAKE, qs=8 * 128, k=FAKE, ks=4 * 128, v=FAKE, vs=4 * 128, qo=FAKE, kp=FAKE, vp=FAKE, table=FAKE, start=FAKE, n=None, pos=None)
    a.update(kw)
    return _lib.load().traj_paged_append(*a.values(), ctypes.byref(sh), theta, None)


def attn(sh=None, scale=0.0, ws=None, ws_bytes=0, **kw):
    sh = sh or shape()
    a = dict(q=FAKE, kp=FAKE, vp=FAKE, table=FAKE, lens=FAKE, n=None, out=FAKE)
    a.update(kw)
    return _lib.load().traj_paged_attn(*a.values(), ctypes.byref(sh), scale, 0, ws, ws_bytes, None)


def test_paged_shapes():
    for bad in BAD_SHAPES:
        assert append(shape(**bad)) == SHAPE, bad
        assert attn(shape(**bad)) == SHAPE, bad
        assert _lib.load().traj_paged_attn_workspace_size(ctypes.byref(shape(**bad))) == 0
    for bad in (dict(D=96), dict(token_stride=(1 << 25) + 8)):
        assert append(shape(**bad)) == UNSUPPORTED and attn(shape(**bad)) == UNSUPPORTED
    for none in (dict(B=0), dict(T=0)):
        assert append(shape(**none), k=None) == 0 and attn(shape(**none), q=None) == 0
        for columns in (4, 4096):
            assert _lib.load().traj_paged_attn_workspace_size(ctypes.byref(shape(max_pages=columns, table_stride=columns, **none))) == 0
    assert _lib.load().traj_paged_attn(*[FAKE] * 7, None, 0.0, 0, None, 0, None) == NULL


def test_append_arguments():
    for name in ("k", "v", "kp", "vp", "table", "start", "q", "qo"):
        assert append(**{name: None}) == NULL, name
    for name in ("q", "k", "v", "qo", "kp", "vp"):
        assert append(**{name: ODD}) == SHAPE, name
    for bad in (dict(qs=8 * 128 - 8), dict(ks=4 * 128 - 8), dict(vs=4 * 128 + 4), dict(ks=4 * 128 + 1)):
        assert append(**bad) == SHAPE, bad
    for theta in (float("nan"), float("inf"), -1.0):
        assert append(theta=theta) == ARG


def test_attention_arguments():
    for name in ("q", "kp", "vp", "table", "lens", "out"):
        assert attn(**{name: None}) == NULL, name
    for name in ("q", "kp", "vp", "out"):
        assert attn(**{name: ODD}) == SHAPE, name
    assert attn(scale=float("nan")) == ARG and attn(scale=float("inf")) == ARG
    # more workgroups than a launch can have
    assert attn(shape(B=65535, T=16, Hq=512, Hkv=512)) == SHAPE
    # many rows fill the chip unsplit
    assert _lib.load().traj_paged_attn_workspace_size(ctypes.byref(shape(B=1024, T=8192, max_pages=4096, table_stride=4096))) == 0
    long = shape(max_pages=4096, table_stride=4096)
    need = _lib.load().traj_paged_attn_workspace_size(ctypes.byref(long))
    assert need > 0
    assert attn(long, ws=FAKE, ws_bytes=need - 1) == WORKSPACE
    assert attn(long, ws=ODD, ws_bytes=need) == WORKSPACE


def test_a_workspace_covers_every_split_of_the_lengths():
    """Ranges of the batch's keys as the device cuts them, for lengths of every kind: never more than the workspace has slots."""
    sizes = _lib.load().traj_paged_attn_workspace_size
    for B, T, Hq, Hkv, columns in ((1, 1, 8, 8, 4000), (7, 1, 4, 1, 300), (300, 2, 2, 2, 50), (3, 64, 4, 1, 1000), (1, 1, 1, 1, 9)):
        sh = shape(B=B, T=T, Hq=Hq, Hkv=Hkv, max_pages=columns, table_stride=columns)
        rows = T * Hq // Hkv
        tile = next(n for n in (16, 32, 64, 128) if rows <= n or n == 128)
        units = Hkv * -(-rows // tile)
        cap = columns * 16
        size = sizes(ctypes.byref(sh))
        if cap <= 256:  # never split
            assert size == 0
            continue
        slots, rest = divmod(size - 8 * B, units * tile * (128 + 2) * 4)
        assert rest == 0
        for lens in ([cap] * B, [cap] + [0] * (B - 1), [1] * B, [129] * B, [(i * 7919) % cap for i in range(B)], [cap // 2] * (B // 2 + 1)):
            work = sum(lens) * units / 128
            chunk = 128 * max(1, math.ceil(max(work / 2048, min(work / 256, 8))))
            assert sum(max(1, -(-n // chunk)) for n in lens) <= max(slots, B), (B, T, lens[:3])


def adjust(sh=None, k=3, logits=FAKE, conf=FAKE, idx=FAKE, ws=None, ws_bytes=0, **kw):
    sh = sh or _lib.LogitsShape(32, 1000, 1000, 0)
    d = dict(rows_per_seq=8, history_size=0, bias_size=0, n_masks=0, mask_stride=0)
    a = _lib.LogitAdjust(**{**d, **kw})
    return _lib.load().traj_confidence_topk_adjusted(logits, k, conf, idx, ctypes.byref(sh), ctypes.byref(a), ws, ws_bytes, None)


def test_adjusted_arguments():
    L = _lib.LogitsShape
    assert adjust(L(4, 100, 100, 9)) == DTYPE
    assert adjust(L(4, 100, 99, 0)) == SHAPE
    assert adjust(k=0) == ARG and adjust(k=9) == ARG and adjust(L(4, 2, 2, 1)) == ARG
    assert adjust(L(4, (1 << 19) + 1, 1 << 21, 0)) == UNSUPPORTED
    for bad in (dict(rows_per_seq=0), dict(history_size=-1), dict(bias_size=-1), dict(history_size=1 << 29, bias_size=1 << 29),
                dict(mask=FAKE, n_masks=0, mask_stride=32), dict(mask=FAKE, n_masks=32, mask_stride=31),
                dict(mask=FAKE, n_masks=31, mask_stride=32)):
        assert adjust(**bad) == SHAPE, bad
    assert adjust(logits=None) == NULL and adjust(conf=None) == NULL and adjust(idx=None) == NULL
    assert adjust(logits=0x1001) == SHAPE and adjust(L(32, 1000, 1000, 1), logits=0x1002) == SHAPE
    assert adjust(history_size=4) == NULL
    assert adjust(bias_size=4, bias_ids=FAKE) == NULL and adjust(bias_size=4, bias=FAKE) == NULL
    assert adjust(history_size=4, history=FAKE) == WORKSPACE
    assert adjust(L(1 << 24, 1000, 1000, 0)) == SHAPE
    assert adjust(L(1 << 22, 1000, 1000, 0), rows_per_seq=1, history_size=4, history=FAKE) == SHAPE
    assert adjust(L(0, 1000, 1000, 0), logits=None, history_size=4) == 0
    lib = _lib.load()
    one = _lib.LogitAdjust(rows_per_seq=8, history_size=4)
    need = lib.traj_confidence_topk_adjusted_workspace_size(ctypes.byref(L(400, 1000, 1000, 0)), 3, ctypes.byref(one))
    assert need > 0 and need % 256 == 0
    assert adjust(L(400, 1000, 1000, 0), history_size=4, history=FAKE, ws=FAKE, ws_bytes=need - 256) == WORKSPACE
    assert adjust(L(400, 1000, 1000, 0), history_size=4, history=FAKE, ws=ODD, ws_bytes=need) == WORKSPACE
    assert lib.traj_confidence_topk_adjusted(FAKE, 3, FAKE, FAKE, None, ctypes.byref(one), None, 0, None) == NULL
    assert lib.traj_confidence_topk_adjusted(FAKE, 3, FAKE, FAKE, ctypes.byref(L(4, 100, 100, 0)), None, None, 0, None) == NULL


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16)
    pages = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        tsp.paged_append(x, x, pages, pages, n[None], n)
    with pytest.raises(TypeError):
        tsp.paged_attn(x, pages, pages, n[None], n)
    with pytest.raises(TypeError):
        tsp.confidence_topk_adjusted(torch.zeros(2, 100), 3, 1)
