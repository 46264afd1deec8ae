"""What the 8-bit calls refuse, before anything reaches the device (CPU only)."""

import ctypes
import os

import pytest
import torch

import paper_2608_27514_amd as tsp
from paper_2608_27514_amd import _lib
from test_gpu_eight import PRODUCT
from test_paged_refusals import BAD_SHAPES, FAKE, NULL, ODD, SHAPE, UNSUPPORTED, WORKSPACE, ARG, shape

pytestmark = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libtrajspec.so not built")


def append(sh=None, sb=16, theta=1e4, **kw):
    sh = sh or shape()
    a = dict(q=FAKE, qs=8 * 128, k=FAKE, ks=4 * 128, v=FAKE, vs=4 * 128, qo=FAKE, kp=FAKE, vp=FAKE, ksc=FAKE + 1, vsc=FAKE + 3, table=FAKE,
             start=FAKE, n=None, pos=None)
    a.update(kw)
    return _lib.load().traj_paged_append_eight(*a.values(), ctypes.byref(sh), sb, theta, None)


def attn(sh=None, sb=16, scale=0.0, ws=None, ws_bytes=0, **kw):
    sh = sh or shape()
    a = dict(q=FAKE, kp=FAKE, vp=FAKE, ksc=FAKE + 1, vsc=FAKE + 3, table=FAKE, lens=FAKE, n=None, out=FAKE)
    a.update(kw)
    return _lib.load().traj_paged_attn_eight(*a.values(), ctypes.byref(sh), sb, scale, 0, ws, ws_bytes, None)


def test_shapes():
    size = _lib.load().traj_paged_attn_eight_workspace_size
    for bad in BAD_SHAPES + [dict(page_stride=16 * 512 + 8), dict(token_stride=520), dict(head_stride=136)]:
        assert append(shape(**bad)) == SHAPE and attn(shape(**bad)) == SHAPE, bad
        assert size(ctypes.byref(shape(**bad)), 16) == 0
    for sb in (0, -1, 5, 32, 17):
        assert append(sb=sb) == SHAPE and attn(sb=sb) == SHAPE and size(ctypes.byref(shape()), sb) == 0
    wide = shape(page_size=128, page_stride=128 * 512)
    assert append(wide, 128) == SHAPE and attn(wide, 128) == SHAPE  # 64 tokens of a scale at most
    assert append(shape(D=96)) == UNSUPPORTED and attn(shape(D=96)) == UNSUPPORTED
    for none in (dict(B=0), dict(T=0)):
        assert append(shape(**none), k=None) == 0 and attn(shape(**none), q=None) == 0
    assert _lib.load().traj_paged_append_eight(*[FAKE, 8, FAKE, 8, FAKE, 8], *[FAKE] * 9, None, 16, 1.0, None) == NULL
    assert _lib.load().traj_paged_attn_eight(*[FAKE] * 9, None, 16, 0.0, 0, None, 0, None) == NULL


def test_append_arguments():
    for name in ("k", "v", "kp", "vp", "ksc", "vsc", "table", "start", "q", "qo"):
        assert append(**{name: None}) == NULL, name
    for name in ("q", "k", "v", "qo", "kp", "vp"):
        assert append(**{name: ODD}) == SHAPE, name
    for bad in (dict(qs=8 * 128 - 8), dict(ks=4 * 128 - 8), dict(vs=4 * 128 + 4)):
        assert append(**bad) == SHAPE, bad
    for theta in (float("nan"), float("inf"), -1.0):
        assert append(theta=theta) == ARG


def test_attention_arguments():
    for name in ("q", "kp", "vp", "ksc", "vsc", "table", "lens", "out"):
        assert attn(**{name: None}) == NULL, name
    for name in ("q", "kp", "vp", "out"):
        assert attn(**{name: ODD}) == SHAPE, name
    assert attn(scale=float("nan")) == ARG and attn(scale=float("inf")) == ARG
    assert attn(shape(B=65535, T=16, Hq=512, Hkv=512)) == SHAPE
    long = shape(max_pages=4096, table_stride=4096)
    need = _lib.load().traj_paged_attn_eight_workspace_size(ctypes.byref(long), 16)
    assert need > 0
    assert attn(long, ws=FAKE, ws_bytes=need - 1) == WORKSPACE and attn(long, ws=ODD, ws_bytes=need) == WORKSPACE


def test_product_arguments():
    lib = _lib.load()
    size = lib.traj_linear_eight_workspace_size

    def linear(M=32, K=256, N=128, x=FAKE, w=FAKE, s=FAKE + 1, y=FAKE, ws=FAKE, ws_bytes=None):
        return lib.traj_linear_eight(x, w, s, y, M, K, N, 0, ws, size(M, K, N) if ws_bytes is None else ws_bytes, None)

    for bad in (dict(M=-1), dict(K=0), dict(K=12), dict(N=4), dict(N=0), dict(N=100), dict(M=1 << 40), dict(K=-8)):
        assert linear(**bad) == SHAPE, bad
        b = {**dict(M=32, K=256, N=128), **bad}
        assert size(b["M"], b["K"], b["N"]) == 0
    for big in (dict(K=65536 + 8), dict(N=(1 << 24) + 8)):
        assert linear(**big) == UNSUPPORTED, big
        assert lib.traj_quantize_eight(FAKE, FAKE, FAKE, big.get("K", 256), big.get("N", 128), None) == UNSUPPORTED
    assert linear(M=0, x=None, ws=None) == 0
    for name in ("x", "w", "s", "y"):
        assert linear(**{name: None}) == NULL, name
    for name in ("x", "w", "y"):
        assert linear(**{name: ODD}) == SHAPE, name
    assert linear(ws=None) == WORKSPACE and linear(ws=ODD) == WORKSPACE and linear(M=1000, ws_bytes=1000 * 256) == WORKSPACE
    for bad in (dict(K=0), dict(K=9), dict(N=12), dict(N=-8)):
        b = {**dict(K=256, N=128), **bad}
        assert lib.traj_quantize_eight(FAKE, FAKE, FAKE, b["K"], b["N"], None) == SHAPE, bad
    for i in range(3):
        a = [FAKE] * 3
        a[i] = None
        assert lib.traj_quantize_eight(*a, 256, 128, None) == NULL
    assert lib.traj_quantize_eight(ODD, FAKE, FAKE, 256, 128, None) == SHAPE and lib.traj_quantize_eight(FAKE, ODD, FAKE, 256, 128, None) == SHAPE


@pytest.mark.parametrize("K,N", [(256, 128), (4096, 12288), (3584, 4608), (72, 8), (65536, 1024)])
def test_a_workspace_for_more_rows_serves_fewer(K, N):
    """What a call needs at least (x in 8 bits and its scales) never exceeds what is reported for more rows."""
    size = _lib.load().traj_linear_eight_workspace_size
    KP = -(-K // 128) * 128
    most = 0
    for M in list(range(1, 300)) + [511, 512, 513, 2000, 4096, 30000]:
        up = lambda n: -(-n // 256) * 256  # noqa: E731
        least = 0 if M <= 16 and M * KP <= 65536 else up(M * KP) + up(-(-M // 128) * KP)  # a few rows need none
        assert size(M, K, N) >= least and least >= most
        most = least


def product_plan(M, K, N):
    """(kernel, k ranges) that a product runs with: 6 tilings, then 3 x 3 kernels of few rows."""
    out = (ctypes.c_int32 * 2)()
    fn = _lib.load().traj_test_gemm_eight_plan
    fn.restype, fn.argtypes = None, [ctypes.c_int64] * 3 + [ctypes.POINTER(ctypes.c_int32)]
    fn(M, K, N, out)
    return tuple(out)


def test_the_tested_products_reach_every_kernel():
    plans = {product_plan(*c) for c in PRODUCT}
    assert {kernel for kernel, _ in plans} == set(range(15))
    assert {kernel for kernel, splits in plans if splits > 1} == set(range(6))
    # a product of the benchmark's layer with many tokens, and few rows of its widest matrix
    assert product_plan(4096, 4096, 12288) == (5, 1) and product_plan(8, 4096, 12288)[0] == 8


def test_the_binding_refuses_host_tensors_and_other_types():
    x = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16)
    pages = torch.zeros(2, 16, 2, 64, dtype=torch.float8_e4m3fn)
    scale = torch.zeros(2, 1, 2, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    n = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        tsp.paged_append8(x, x, pages, pages, scale, scale, n[None], n)
    with pytest.raises(TypeError):
        tsp.paged_attn8(x, pages, pages, scale, scale, n[None], n)
    with pytest.raises(TypeError):
        tsp.quantize8(torch.zeros(128, 128, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        tsp.linear8(torch.zeros(1, 128, dtype=torch.bfloat16), torch.zeros(2, 128, 64, dtype=torch.float8_e4m3fn), scale)
