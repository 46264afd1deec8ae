"""GPU parity: caches and weights in 8 bits against their oracle.

A rounding to e4m3 is off by at most half a step: 2^-4 of the value, or 2^-10 of the scale among the subnormals.  Values and
weights are bf16 and taken to 8 bits directly, so they match bit for bit.  Keys are rotated in fp32 first, whose products with a
sine and a cosine are off by e = 2^-20 (|a| + |b|): |err| <= 2^-4 (|y| + e) + 2^-10 scale + e.
Attention: keys and values enter exactly; fp32 scores (128 products each), weights to 2^-16 and sums over some thousand
keys move the result by less than 2^-10 sum w |v|, its own rounding to bf16 by 2^-8 |out|.
Product: operands enter exactly, the matrix core adds 8 products at a time, each cut to 2^-13 of the
largest (8 2^-13 = 2^-10 of the sum of magnitudes), and those sums in fp32; the result is rounded to
bf16 (2^-8 of it)."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import cuda
from oracle import eight
from oracle.layer import bf16_round

pytestmark = pytest.mark.gpu
BF, E4, E8, U8 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.uint8


def bf(x):
    return cuda(np.asarray(x, dtype=np.float32), BF)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def normal(rng, *shape):
    return bf16_round(rng.standard_normal(shape))


def i32(x):
    return cuda(np.asarray(x, dtype=np.int32))


def e4(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(E4).cuda()


def e8(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.uint8)).view(E8).cuda()


def bytes_of(t):
    return t.view(U8).cpu().numpy().astype(np.int64)


def heads_first(x):
    """The same pool with its memory as [pages, Hkv, page_size, D]."""
    return x.view(U8).transpose(1, 2).contiguous().transpose(1, 2).view(E4)


def make_table(rng, B, columns, spare=3):
    pages = B * columns + spare
    return rng.permutation(pages)[:B * columns].reshape(B, columns).astype(np.int32), pages


def make_pools(rng, pages, ps, sb, H, D):
    byte = rng.integers(118, 122, (2, pages, ps // sb, H))
    return [*eight.e4m3(np.clip(100 * rng.standard_normal((2, pages, ps, H, D)), -448, 448)), *byte]


def on_gpu(pools, layout=lambda x: x):
    return layout(e4(pools[0])), layout(e4(pools[1])), e8(pools[2]), e8(pools[3])


def check_append(got, q_out, want, pools, exact, inputs, theta):
    """The call's pools and q_out against the oracle's; inputs: (q, k) before rotation."""
    ref, size = want
    e = 2.0 ** -20 * size
    if q_out is not None:
        assert (np.abs(f64(q_out) - ref) <= 2.0 ** -8 * (np.abs(ref) + e) * (e > 0) * (theta > 0) + e).all()
    for i, name in ((2, "k_scale"), (3, "v_scale")):
        assert np.array_equal(bytes_of(got[i]), pools[i]), name
    assert np.array_equal(f64(got[1]), pools[1])
    written = ~np.isnan(exact[0])
    k = f64(got[0])
    assert np.array_equal(k[~written], pools[0][~written])
    s = np.broadcast_to(eight.scale_value(pools[2]).repeat(k.shape[1] // pools[2].shape[1], 1)[..., None], k.shape)[written]
    y = exact[0][written]
    e = 2.0 ** -20 * 2 * np.abs(inputs).max() * (theta > 0)
    err = np.abs(k[written] * s - y)
    assert (err <= 2.0 ** -4 * (np.abs(y) + e) + 2.0 ** -10 * s + e).all()
    assert (k[written] != pools[0][written]).mean() <= 1e-3  # only next to the middle between two codes


APPEND = [
    # B, T, Hq, Hkv, D, page_size, scale block, start, n_new, pos0
    (1, 1, 4, 4, 64, 16, 16, [5], None, None),
    (1, 1, 32, 8, 128, 16, 16, [40], None, [100000]),
    (3, 7, 28, 4, 128, 5, 5, [0, 3, 11], [7, 0, 4], [0, 9, 250000]),
    (2, 33, 8, 1, 64, 1, 1, [2, 0], None, None),
    (4, 300, 4, 2, 128, 48, 24, [0, 17, 47, 48], [300, 299, 1, 150], [5, 6, 7, 1000]),
    (2, 600, 2, 2, 64, 32, 32, [0, 31], [600, 13], None),
    (3, 130, 6, 3, 128, 128, 64, [63, 64, 1], [130, 64, 127], None),
    (2, 70, 3, 3, 64, 49, 49, [48, 20], None, [7, 7]),
    (2, 50, 4, 2, 128, 21, 7, [6, 15], [50, 1], None),
    (5, 3, 2, 1, 64, 256, 8, [255, 7, 8, 0, 500], [3, 2, 1, 0, 3], None),
    (64, 1, 4, 4, 128, 16, 16, list(range(64)), None, None),
]


@pytest.mark.parametrize("B,T,Hq,Hkv,D,ps,sb,start,n_new,pos0", APPEND)
@pytest.mark.parametrize("theta", [500000.0, 0.0])
def test_append_parity(B, T, Hq, Hkv, D, ps, sb, start, n_new, pos0, theta):
    rng = np.random.default_rng(B * 1000 + T)
    # rows of very different sizes, so that scales differ and grow
    qkv = bf16_round(rng.standard_normal((B, T, (Hq + 2 * Hkv) * D)) * 2.0 ** rng.integers(-3, 4, (B, T, 1)))
    columns = -(-(max(start) + T) // ps)
    table, pages = make_table(rng, B, columns)
    before = make_pools(rng, pages, ps, sb, Hkv, D)
    q0 = normal(rng, B, T, Hq, D)  # what q_out holds before
    q, k, v = (x.reshape(B, T, -1, D) for x in np.split(qkv, [Hq * D, (Hq + Hkv) * D], axis=-1))
    ref, pools, exact = eight.paged_append8(q, k, v, before, table, start, n_new, pos0, theta, q_out=q0)
    size = eight.paged_append8(np.abs(q) + np.abs(np.roll(q, D // 2, -1)), k, v, before, table, start, n_new, pos0, 0, q_out=0 * q0)[0]
    qg, kg, vg = (x.view(B, T, -1, D) for x in bf(qkv).split([Hq * D, Hkv * D, Hkv * D], -1))
    got = on_gpu(before, heads_first if B % 2 else lambda x: x)
    out = bf(q0)
    opt = lambda x: None if x is None else i32(x)  # noqa: E731
    assert tsp.paged_append8(kg, vg, *got, i32(table), i32(start), q=qg, q_out=out, n_new=opt(n_new), pos0=opt(pos0), rope_theta=theta) is out
    assert tsp.device_status() == 0
    check_append(got, out, (ref, size), pools, exact, qkv, theta)


@pytest.mark.parametrize("D,ps,sb", [(128, 16, 16), (64, 24, 8), (128, 64, 64), (64, 48, 24), (128, 32, 1), (128, 60, 5), (64, 64, 32)])
def test_append_from_every_offset(D, ps, sb):
    """A sequence for each place of a page to begin at, calls shorter and longer than a group of rows."""
    rng = np.random.default_rng(D + ps + sb)
    for T in (1, 7, 16, 17, 33, 70):
        columns = -(-(ps + T) // ps)
        table, pages = make_table(rng, ps, columns)
        before = make_pools(rng, pages, ps, sb, 1, D)
        k, v = (bf16_round(rng.standard_normal((ps, T, 1, D)) * 2.0 ** rng.integers(-3, 4, (ps, T, 1, 1))) for _ in range(2))
        start, n_new = np.arange(ps, dtype=np.int32), rng.integers(0, T + 1, ps).astype(np.int32)
        _, pools, _ = eight.paged_append8(k, k, v, before, table, start, n_new, theta=0)
        got = on_gpu(before)
        tsp.paged_append8(bf(k), bf(v), *got, i32(table), i32(start), n_new=i32(n_new), rope_theta=0.0)
        assert tsp.device_status() == 0
        for x, want in zip(got, pools):
            assert np.array_equal(f64(x) if x.dtype == E4 else bytes_of(x), want)


def test_append_token_by_token_and_again():
    """Single tokens into blocks whose scales grow, and a denoising step that writes its rows a second time."""
    rng = np.random.default_rng(1)
    B, T, H, D, ps, sb = 2, 40, 2, 128, 32, 16
    table, pages = make_table(rng, B, 3)
    pools = make_pools(rng, pages, ps, sb, H, D)
    k, v = (bf16_round(rng.standard_normal((B, T, H, D)) * 2.0 ** rng.integers(-4, 5, (B, T, 1, 1))) for _ in range(2))
    got = on_gpu(pools)
    for t in range(T):
        start = np.array([t, t + 3])
        _, pools, _ = eight.paged_append8(None, k[:, t:t + 1], v[:, t:t + 1], pools, table, start, theta=0)
        assert tsp.paged_append8(bf(k[:, t:t + 1]), bf(v[:, t:t + 1]), *got, i32(table), i32(start), rope_theta=0.0) is None
    for n in range(2):
        _, pools, _ = eight.paged_append8(None, k[:, :9] * (n + 1), v[:, :9], pools, table, [20, 33], theta=0)
        tsp.paged_append8(bf(k[:, :9] * (n + 1)), bf(v[:, :9]), *got, i32(table), i32([20, 33]), rope_theta=0.0)
    for x, want in zip(got, pools):
        assert np.array_equal(f64(x) if x.dtype == E4 else bytes_of(x), want)


def test_append_values_at_the_edges():
    """Zeros, the largest and smallest values, infinities and NaN; scale bytes that no call writes."""
    H, D, ps = 1, 64, 8
    x = np.zeros((1, 8, H, D))
    x[0, 1, 0, :4] = 3.0e38, -3.0e38, 1.0, 1.0e-30
    x[0, 2, 0, :2] = 448.0, 448.0 * 2.0 ** -9
    x[0, 3, 0, :3] = 450.0, np.nan, np.inf
    x[0, 4, 0, :2] = 2.0 ** -130, -2.0 ** -109
    x = bf16_round(x)
    table = np.array([[0]], np.int32)
    for sb in (1, 8):
        for old in (0, 255, 130):
            zero = [np.zeros((1, ps, H, D)), np.ones((1, ps, H, D)), np.full((1, ps // sb, H), old), np.full((1, ps // sb, H), old)]
            for start in (0, 3):
                _, want, _ = eight.paged_append8(None, x[:, start:], x[:, start:], zero, table, [start], theta=0)
                got = on_gpu(zero)
                tsp.paged_append8(bf(x[:, start:]), bf(x[:, start:]), *got, i32(table), i32([start]), rope_theta=0.0)
                for a, b in zip(got, want):
                    a = f64(a) if a.dtype == E4 else bytes_of(a)
                    assert np.array_equal(a, b, equal_nan=True), (sb, old, start)


def test_append_skips_what_has_no_place():
    rng = np.random.default_rng(4)
    B, T, H, D, ps, sb = 4, 5, 2, 64, 4, 2
    k, v, q = normal(rng, B, T, H, D), normal(rng, B, T, H, D), normal(rng, B, T, H, D)
    table = np.array([[0, 1, 2], [3, -1, 4], [5, 6, 99], [7, 8, 9]], np.int32)
    start, n_new = [9, 3, 6, -3], [5, 5, 9, -2]
    before = make_pools(rng, 10, ps, sb, H, D)
    ref, pools, _ = eight.paged_append8(q, k, v, before, table, start, n_new, theta=0)
    got = on_gpu(before)
    tsp.device_status()
    out = tsp.paged_append8(bf(k), bf(v), *got, i32(table), i32(start), q=bf(q), n_new=i32(n_new), rope_theta=0.0)
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH | tsp.DEV_BAD_PAGE
    assert np.array_equal(f64(out), ref)
    for x, want in zip(got, pools):
        assert np.array_equal(f64(x) if x.dtype == E4 else bytes_of(x), want)


# ---------------------------------------------------------------- attention

def attend(rng, B, T, Hq, Hkv, D, ps, sb, lens, causal, layout=lambda x: x, scale=0.0, sharp=1.0, n_new=None):
    """Runs a call on a pool whose unused rows are NaN, unused scales too, and compares it; returns the device tensors."""
    cap = max(1, -(-max(lens) // ps))
    table, pages = make_table(rng, B, cap)
    pools = make_pools(rng, pages, ps, sb, Hkv, D)
    q = bf16_round(sharp * rng.standard_normal((B, T, Hq, D)))
    used = np.zeros((pages, ps), bool)
    for b, n in enumerate(lens):
        s = np.arange(n)
        used[table[b, s // ps], s % ps] = True
        table[b, -(-n // ps):] = -1
    kp, vp = (eight.paged_values(pools[i], pools[2 + i]) for i in (0, 1))
    ref, weight = oracle.paged_attention(q, kp, vp, table, lens, causal, scale or None, n_new=n_new)
    pools[0][~used] = pools[1][~used] = np.nan
    idle = ~used.reshape(pages, -1, sb).any(2)
    pools[2][idle], pools[3][idle] = 255, rng.integers(0, 256, pools[3][idle].shape)
    t = (bf(q), *on_gpu(pools, layout), i32(table), i32(lens))
    out = tsp.paged_attn8(*t, causal=causal, scale=scale, n_new=None if n_new is None else i32(n_new))
    assert tsp.device_status() == 0
    err = np.abs(f64(out) - ref)
    tol = 2.0 ** -10 * weight + 2.0 ** -8 * np.abs(ref) + 1e-30
    assert (err <= tol).all(), float((err - tol).max())
    return t, out


ATTEND = [
    # T, Hq, Hkv, D, page_size, scale block, lens
    (1, 4, 4, 64, 16, 16, [192]),
    (1, 2, 2, 128, 32, 8, [0, 1, 31, 32, 33, 127, 128, 129, 300]),
    (1, 16, 1, 64, 64, 64, [1000, 77, 0, 5]),
    (1, 17, 1, 128, 16, 1, [100, 260]),                  # 17 rows: a second fragment of one row
    (3, 14, 2, 128, 24, 8, [500, 2, 3, 0, 129]),          # causal: rows before the sequence's start see nothing
    (5, 4, 4, 64, 5, 5, [777, 4, 131]),
    (32, 4, 1, 128, 1, 1, [200, 33]),
    (64, 2, 2, 64, 736, 46, [736, 64, 65, 100]),
    (33, 1, 1, 128, 48, 24, [400]),
    (2, 8, 2, 64, 100, 50, [4000, 1]),                    # one long sequence: split over many workgroups
    (1, 8, 8, 128, 64, 64, [5000, 40, 2222]),
    (4, 8, 1, 128, 48, 3, [3000]),
    (4, 8, 1, 64, 80, 20, [2900, 100]),
    (32, 8, 2, 128, 16, 16, [1500, 300]),                 # 128 rows, split
    (16, 8, 2, 128, 20, 4, [900, 90]),
    (40, 8, 2, 128, 12, 6, [513, 31, 0]),                 # two row tiles that share the keys, the second of 32 rows
    (48, 12, 4, 64, 32, 32, [700, 0, 64]),                # heads in pairs
    (3, 9, 3, 64, 16, 16, [600, 257]),                    # and an odd number of them
    (1, 6, 3, 64, 48, 16, [1, 2000]),
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,ps,sb,lens", ATTEND)
def test_attention_parity(T, Hq, Hkv, D, ps, sb, lens, causal):
    attend(np.random.default_rng(T + ps), len(lens), T, Hq, Hkv, D, ps, sb, lens, causal)


def test_attention_layouts_scales_and_many_sequences():
    rng = np.random.default_rng(8)
    for ps, sb in ((16, 16), (20, 4), (64, 32)):
        attend(rng, 3, 2, 8, 4, 128, ps, sb, [90, 400, 1], True, layout=heads_first, scale=0.3)
    attend(rng, 2, 1, 4, 2, 64, 16, 16, [1500, 40], False, sharp=8.0)  # peaked weights: the maximum moves often
    lens = rng.integers(0, 90, 150)
    lens[[3, 64, 149]] = 3000, 0, 1111
    attend(rng, 150, 1, 2, 1, 64, 16, 16, lens.tolist(), False)
    attend(rng, 3, 7, 4, 2, 128, 16, 16, [27, 300, 9], True, n_new=[7, 0, 3])


@pytest.mark.parametrize("T", [2, 6, 10, 20, 40])
def test_attention_padding_may_hold_anything(T):
    """Queries behind n_new are NaN: their rows are 0 and no other row changes; rows that see nothing are 0 too."""
    rng = np.random.default_rng(T)
    n_new = [T, T // 2, 0, 1]
    for ps, sb, lens in ((16, 8, [40, 200, 33, 0]), (20, 20, [900, 30, 70, 5])):  # whole, split
        (q, *t), out = attend(rng, 4, T, 8, 2, 128, ps, sb, lens, True, n_new=n_new)
        for b, n in enumerate(n_new):
            assert not out[b, n:].any()
            q[b, n:] = float("nan")
        assert torch.equal(tsp.paged_attn8(q, *t, causal=True, n_new=i32(n_new)), out)


def test_attention_lengths_around_every_tile():
    """A sequence of every length up to two rounds of tiles, whole and within a batch that is split."""
    rng = np.random.default_rng(9)
    lens = list(range(0, 530))
    attend(rng, len(lens), 1, 2, 1, 64, 16, 8, lens, False)
    attend(rng, len(lens), 1, 1, 1, 128, 12, 4, lens, False)
    lens = list(range(0, 270))
    attend(rng, len(lens), 9, 4, 1, 64, 16, 16, lens, True)
    attend(rng, len(lens), 30, 3, 1, 128, 10, 5, lens, True)


def test_attention_unsplit_and_in_a_larger_workspace_agree():
    rng = np.random.default_rng(10)
    import ctypes
    from paper_2608_27514_amd import _lib
    t, out = attend(rng, 2, 2, 8, 2, 128, 32, 16, [3000, 700], False)
    q, kp, vp, ks, vs, table, lens = t
    sh = _lib._paged_struct(*_lib._paged_sizes(2, 2, 8, kp, vp, table, 0, E4))[0]
    whole = torch.empty_like(q)
    ptr = [x.data_ptr() for x in (q, kp, vp, ks, vs, table, lens)] + [None, whole.data_ptr()]
    assert tsp.load().traj_paged_attn_eight(*ptr, ctypes.byref(sh), 16, 0.0, 0, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    # both are within the tolerance above of the same value; |out| and the weighted sums stay below 8
    assert (whole.float() - out.float()).abs().max().item() <= 2 * 8 * (2.0 ** -10 + 2.0 ** -8)
    need = tsp.paged_attn8_workspace_size(q, kp, vp, ks, vs, table)
    assert need > 0
    big = torch.full((need + 4096,), 255, dtype=U8, device="cuda")  # NaN in every float
    assert torch.equal(tsp.paged_attn8(*t, workspace=big), out)
    assert (big[need:] == 255).all()


def test_attention_bad_lengths_and_pages():
    rng = np.random.default_rng(11)
    B, T, H, D, ps, sb = 3, 1, 2, 64, 16, 8
    table = np.array([[0, 1], [2, 77], [-1, 3]], np.int32)
    pools = make_pools(rng, 4, ps, sb, H, D)
    q = normal(rng, B, T, H, D)
    kp, vp = (eight.paged_values(pools[i], pools[2 + i]) for i in (0, 1))
    lens = [1000, 30, 20]
    for page in (16, 8):  # the same pool in pages within a tile's blocks, and smaller ones
        f = ps // page
        k8, v8 = kp.reshape(-1, page, H, D), vp.reshape(-1, page, H, D)
        t8 = np.where((table >= 0) & (table < 4), table, -99)[:, :, None] * f + np.arange(f) if f > 1 else table[:, :, None]
        t8 = t8.reshape(B, -1).astype(np.int32)
        ref, weight = oracle.paged_attention(q, k8, v8, t8, lens)
        got = [x.view(U8).reshape(4 * f, -1, *x.shape[2:]).view(x.dtype) for x in on_gpu(pools)]
        tsp.device_status()
        out = tsp.paged_attn8(bf(q), *got, i32(t8), i32(lens))
        assert tsp.device_status() == tsp.DEV_BAD_LENGTH | tsp.DEV_BAD_PAGE
        assert (np.abs(f64(out) - ref) <= 2.0 ** -10 * weight + 2.0 ** -8 * np.abs(ref) + 1e-30).all()
    out = tsp.paged_attn8(bf(q), *on_gpu(pools), i32(table), i32([-5, 0, -1]))
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH
    assert not out.any()


def test_offsets_past_32_bits():
    """A pool of more than 2^32 values: its last pages are written and read."""
    rng = np.random.default_rng(12)
    ps, sb, Hkv, D, T = 64, 16, 8, 128, 3
    pages = (2 ** 32 + 2 ** 27) // (ps * Hkv * D)
    got = (*(torch.empty(pages, ps, Hkv, D, dtype=E4, device="cuda") for _ in range(2)),
           *(torch.empty(pages, ps // sb, Hkv, dtype=E8, device="cuda") for _ in range(2)))
    n = 2 * ps + 10
    k, v, q = normal(rng, 1, n, Hkv, D), normal(rng, 1, n, Hkv, D), normal(rng, 1, T, Hkv, D)
    table = i32([[pages - 1, pages - 3, 0]])
    tsp.paged_append8(bf(k), bf(v), *got, table, i32([0]), rope_theta=0.0)
    out = tsp.paged_attn8(bf(q), *got, table, i32([n]))
    small = np.arange(3, dtype=np.int32)[None]
    _, pools, _ = eight.paged_append8(None, k, v, make_pools(rng, 3, ps, sb, Hkv, D), small, [0], theta=0)
    kp, vp = (eight.paged_values(pools[i], pools[2 + i]) for i in (0, 1))
    ref, weight = oracle.paged_attention(q, kp, vp, small, [n])
    assert (np.abs(f64(out) - ref) <= 2.0 ** -10 * weight + 2.0 ** -8 * np.abs(ref)).all()
    assert np.array_equal(f64(got[0][pages - 1]), pools[0][0]) and np.array_equal(bytes_of(got[3][pages - 3]), pools[3][1])


def test_empty_batches_do_nothing():
    kp = torch.zeros(2, 16, 2, 64, dtype=E4, device="cuda")
    ks = torch.full((2, 1, 2), 127, dtype=U8, device="cuda").view(E8)
    for B, T in ((0, 3), (2, 0)):
        x = torch.zeros(B, T, 2, 64, dtype=BF, device="cuda")
        table, n = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        assert tsp.paged_append8(x, x, kp, kp.clone(), ks, ks.clone(), table, n, q=x).shape == x.shape
        assert tsp.paged_attn8(x, kp, kp, ks, ks, table, n).shape == x.shape


# ---------------------------------------------------------------- weights and products

def slabs(values):
    """Oracle values [KP, N] in the layout of quantize8."""
    return np.ascontiguousarray(values.reshape(-1, 64, values.shape[1]).transpose(0, 2, 1))


@pytest.mark.parametrize("K,N", [(8, 8), (128, 128), (136, 264), (1000, 712), (64, 1000), (3584, 512), (520, 4608)])
def test_quantised_weights_bit_for_bit(K, N):
    rng = np.random.default_rng(K + N)
    w = bf16_round(rng.standard_normal((K, N)) * 2.0 ** rng.integers(-12, 3, (K, 1)))
    w[0, 0] = 0
    if K > 500:
        w[300, 5], w[301, 6], w[302, 7] = np.nan, np.inf, -np.inf
        w[:128, :128] = 0
    values, byte = eight.quantize8(w)
    w8, scale = tsp.quantize8(bf(w))
    assert w8.shape == (-(-K // 128) * 2, N, 64) and scale.shape == (-(-N // 128), -(-K // 128))
    assert np.array_equal(bytes_of(scale), byte.T)
    assert np.array_equal(f64(w8), slabs(values), equal_nan=True)


def product(rng, M, K, N, accumulate=False, **kw):
    x = bf16_round(rng.standard_normal((M, K)) * 2.0 ** rng.integers(-3, 4, (M, 1)))
    x[:, rng.integers(0, K)] *= 32
    values, byte = eight.quantize8(bf16_round(rng.standard_normal((K, N)) * 2.0 ** rng.integers(-3, 4, (1, N))))
    w8, scale = e4(slabs(values)), e8(byte.T)
    ref, size = eight.linear8(x, values, byte)
    y0 = normal(rng, M, N)
    y = bf(y0) if accumulate else None
    out = tsp.linear8(bf(x), w8, scale, y=y, accumulate=accumulate, **kw)
    if accumulate:
        assert out is y
        ref = ref + y0
    err = np.abs(f64(out) - ref)
    tol = 2.0 ** -10 * size + 2.0 ** -8 * np.abs(ref)
    assert out.dtype == BF and (err <= tol).all(), (M, K, N, float((err - tol).max()))
    return bf(x), w8, scale, out


PRODUCT = [
    # M, K, N
    (1, 8, 8), (1, 128, 128), (1, 4096, 512), (2, 136, 264), (3, 1000, 712), (7, 3584, 1160), (8, 256, 4096), (15, 640, 136), (16, 4096, 1024),
    (17, 512, 520), (31, 128, 1000), (32, 2048, 2048), (33, 1032, 128), (48, 3584, 512), (64, 1024, 1024), (65, 384, 328), (96, 3584, 640),
    (100, 4096, 256), (128, 2048, 1024), (129, 136, 264), (200, 10752, 136), (256, 1024, 4096), (300, 520, 2056), (513, 640, 1000),
    (1000, 256, 8), (2048, 384, 4104), (4096, 136, 4096), (1, 65536, 64), (40, 33000, 72),
    (2, 640, 4112), (16, 384, 8200), (3, 256, 12328), (16, 8192, 136), (5, 16384, 4200), (9, 8320, 8216), (17, 640, 5000), (32, 512, 8296),
    (31, 9000, 200), (70, 4096, 2048), (160, 4096, 6000), (700, 1024, 2048), (1100, 512, 5000), (1300, 2048, 4360),
    (67, 2384, 2360), (66, 4664, 2736), (66, 4968, 2848), (96, 5264, 8416), (449, 2184, 8320), (129, 11472, 5456),
    (3055, 136, 8464), (2340, 680, 5656), (131, 14232, 8232),
]


@pytest.mark.parametrize("M,K,N", PRODUCT)
@pytest.mark.parametrize("accumulate", [False, True])
def test_product_parity(M, K, N, accumulate):
    product(np.random.default_rng(M + K + N), M, K, N, accumulate)


def test_every_number_of_rows():
    """Each count up to past two fragments, over a shape that is split and one that is not."""
    rng = np.random.default_rng(2)
    for M in range(1, 140, 1):
        product(rng, M, 1152 if M % 2 else 128, 264)


def test_product_in_larger_and_smaller_workspaces():
    rng = np.random.default_rng(3)
    for M, K, N in ((20, 4096, 256), (9, 12288, 128), (96, 3584, 640), (300, 4096, 512)):
        need = tsp.linear8_workspace_size(M, K, N)
        big = torch.full((need + 512,), 255, dtype=U8, device="cuda")
        x, w8, scale, out = product(rng, M, K, N, workspace=big)
        assert (big[need:] == 255).all()
        assert torch.equal(tsp.linear8(x, w8, scale), out)
        more = torch.full((tsp.linear8_workspace_size(M + 700, K, N),), 255, dtype=U8, device="cuda")
        product(rng, M, K, N, workspace=more)
        least = -(-M * K // 256) * 256 + -(-(-(-M // 128) * K) // 256) * 256  # x in 8 bits and its scales, nothing else
        tight = torch.full((least + 256,), 255, dtype=U8, device="cuda")
        tsp.linear8(x, w8, scale, workspace=tight[:least])
        product(rng, M, K, N, workspace=tight[:least])
        assert (tight[least:] == 255).all()
        with pytest.raises(tsp.TrajSpecError):
            tsp.linear8(x, w8, scale, workspace=tight[:least - 256])


def test_rows_that_are_not_finite_stay_apart():
    rng = np.random.default_rng(4)
    for M in (3, 40, 300):
        x, w8, scale, out = product(rng, M, 640, 264)
        bad = x.clone()
        bad[1, 7], bad[2, 600], bad[0, 5] = float("nan"), float("inf"), -float("inf")
        y = tsp.linear8(bad, w8, scale)
        assert y[:3].isnan().all() and torch.equal(y[3:], out[3:])
        bad[:3] = 0
        y = tsp.linear8(bad, w8, scale)
        assert not y[:3].any() and torch.equal(y[3:], out[3:])


def test_quantised_weights_times_activations():
    """quantize8 and linear8 together, near the bf16 product of the same matrices."""
    rng = np.random.default_rng(5)
    x, w = normal(rng, 2, 3, 512), normal(rng, 512, 256)
    y = f64(tsp.linear8(bf(x), *tsp.quantize8(bf(w))))
    assert y.shape == (2, 3, 256)
    # both operands are off by half a step each: 2^-4 (and 2^-8 of that) of every product's magnitude, and the subnormals' share
    size = np.abs(x) @ np.abs(w)
    assert (np.abs(y - x @ w) <= (2 * 2.0 ** -4 + 2.0 ** -7) * size + 1.0).all()
    assert tsp.linear8(torch.zeros(0, 512, dtype=BF, device="cuda"), *tsp.quantize8(bf(w))).shape == (0, 256)
