"""GPU parity: the paged key-value cache against its oracle.

Append: the result is rounded once to bf16 (half a step: 2^-8 relative) from fp32 products of values with a
sine and a cosine that are off by at most some 2^-22 each (the angle's fraction of a turn is rounded to fp32:
2 pi 2^-25; the functions' last bits), so |err| <= 2^-8 (|y| + e) + e with e = 2^-20 (|a| + |b|).
Attention: weights rounded to bf16 before the product with V move the result by at most 2^-8 sum w |v|, its own
rounding by 2^-8 |out|; fp32 scores (128 products each) and sums over some thousand keys by less than 2^-10
sum w |v|."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import cuda
from oracle.layer import bf16_round

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
HALF_STEP = 2.0 ** -8


def bf(x):
    return cuda(np.asarray(x, dtype=np.float32), BF)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def normal(rng, *shape):
    return bf16_round(rng.standard_normal(shape))


def i32(x):
    return cuda(np.asarray(x, dtype=np.int32))


def make_table(rng, B, columns, spare=3):
    pages = B * columns + spare
    return rng.permutation(pages)[:B * columns].reshape(B, columns).astype(np.int32), pages


def heads_first(x):
    """The same pool with its memory as [pages, Hkv, page_size, D]."""
    return x.transpose(1, 2).contiguous().transpose(1, 2)


# ---------------------------------------------------------------- append

APPEND = [
    # B, T, Hq, Hkv, D, page_size, start, n_new, pos0
    (1, 1, 4, 4, 64, 16, [5], None, None),
    (1, 1, 32, 8, 128, 16, [40], None, [100000]),
    (3, 7, 28, 4, 128, 5, [0, 3, 11], [7, 0, 4], [0, 9, 250000]),
    (2, 33, 8, 1, 64, 1, [2, 0], None, None),
    (4, 300, 4, 2, 128, 48, [0, 17, 47, 48], [300, 299, 1, 150], [5, 6, 7, 1000]),
    (2, 600, 2, 2, 64, 32, [0, 31], [600, 13], None),
]


@pytest.mark.parametrize("B,T,Hq,Hkv,D,ps,start,n_new,pos0", APPEND)
@pytest.mark.parametrize("theta", [500000.0, 0.0])
def test_append_parity(B, T, Hq, Hkv, D, ps, start, n_new, pos0, theta):
    rng = np.random.default_rng(B * 1000 + T)
    qkv = normal(rng, B, T, (Hq + 2 * Hkv) * D)
    columns = -(-(max(start) + T) // ps)
    table, pages = make_table(rng, B, columns)
    kp, vp = normal(rng, pages, ps, Hkv, D), normal(rng, pages, ps, Hkv, D)
    q0 = normal(rng, B, T, Hq, D)  # what q_out holds before
    parts = np.split(qkv, [Hq * D, (Hq + Hkv) * D], axis=-1)
    q, k, v = (x.reshape(B, T, -1, D) for x in parts)
    ref = oracle.paged_append(q, k, v, kp, vp, table, start, n_new, pos0, theta, q_out=q0)
    big = oracle.paged_append(np.abs(q) + np.abs(np.roll(q, D // 2, -1)), np.abs(k) + np.abs(np.roll(k, D // 2, -1)), v, 0 * kp, 0 * vp,
                              table, start, n_new, pos0, 0, q_out=0 * q0)
    g = bf(qkv)
    qg, kg, vg = (x.view(B, T, -1, D) for x in g.split([Hq * D, Hkv * D, Hkv * D], -1))
    pools = [bf(kp), heads_first(bf(vp))] if B % 2 else [heads_first(bf(kp)), bf(vp)]
    if pools[0].stride() != pools[1].stride():
        pools = [heads_first(p) if B % 2 else p.contiguous() for p in pools]
    out = bf(q0)
    opt = lambda x: None if x is None else i32(x)  # noqa: E731
    got = tsp.paged_append(kg, vg, *pools, i32(table), i32(start), q=qg, q_out=out, n_new=opt(n_new), pos0=opt(pos0), rope_theta=theta)
    assert got is out
    assert tsp.device_status() == 0
    for name, x, r, s in zip(("q", "k"), (out, pools[0]), ref, big):
        e = 2.0 ** -20 * s
        err = np.abs(f64(x) - r)
        over = err - (HALF_STEP * (np.abs(r) + e) * (e > 0) * (theta > 0) + e)
        assert over.max() <= 0, name
    assert np.array_equal(f64(pools[1]), ref[2])  # values are copied; rows not written are as they were


def test_append_in_place_without_queries_and_over_a_contiguous_cache():
    rng = np.random.default_rng(3)
    B, T, Hq, Hkv, D, S = 2, 6, 4, 2, 128, 50
    k, v, q = normal(rng, B, T, Hkv, D), normal(rng, B, T, Hkv, D), normal(rng, B, T, Hq, D)
    cache = bf(normal(rng, B, S, Hkv, D)), bf(normal(rng, B, S, Hkv, D))
    before = [c.clone() for c in cache]
    table = i32(np.arange(B)[:, None])  # a [B, S, Hkv, D] cache is a pool of B pages of S tokens
    start = i32([10, 44])
    assert tsp.paged_append(bf(k), bf(v), *cache, table, start) is None
    qg = bf(q)
    tsp.paged_append(bf(k), bf(v), *cache, table, start, q=qg, q_out=qg)
    want = tsp.paged_append(bf(k), bf(v), *(c.clone() for c in cache), table, start, q=bf(q))
    assert torch.equal(qg, want)
    for b, s in enumerate((10, 44)):
        assert torch.equal(cache[1][b, s:s + T], bf(v)[b])
        for c, c0 in zip(cache, before):
            assert torch.equal(c[b, :s], c0[b, :s]) and torch.equal(c[b, s + T:], c0[b, s + T:])


def test_append_far_positions_keep_their_phase():
    """cos and sin of position 2^20 and of 2^30: exact reduction, which an fp32 angle would miss."""
    D, pos = 64, 2 ** 30
    x = np.zeros((1, 2, 1, D))
    x[..., :D // 2] = 1.0
    kp = torch.zeros(1, 16, 1, D, dtype=BF, device="cuda")
    vp = torch.zeros_like(kp)
    tsp.paged_append(bf(x), bf(x), kp, vp, i32([[0]]), i32([0]), pos0=i32([pos]))
    ref = oracle.rotate(x, np.array([[pos, pos + 1]]), 500000.0)
    # the oracle's own angle is off by 2^30 2^-53
    assert (np.abs(f64(kp)[0, :2] - ref[0]) <= HALF_STEP * np.abs(ref[0]) + 2.0 ** -20).all()


def test_append_skips_what_has_no_place():
    rng = np.random.default_rng(4)
    B, T, Hkv, D, ps = 4, 5, 2, 64, 4
    k, v, q = normal(rng, B, T, Hkv, D), normal(rng, B, T, Hkv, D), normal(rng, B, T, Hkv, D)
    table = np.array([[0, 1, 2], [3, -1, 4], [5, 6, 99], [7, 8, 9]], np.int32)
    start, n_new = [9, 2, 6, -3], [5, 5, 9, -2]
    kp, vp = normal(rng, 10, ps, Hkv, D), normal(rng, 10, ps, Hkv, D)
    ref = oracle.paged_append(q, k, v, kp, vp, table, start, n_new)
    tsp.device_status()
    pools = bf(kp), bf(vp)
    out = tsp.paged_append(bf(k), bf(v), *pools, i32(table), i32(start), q=bf(q), n_new=i32(n_new))
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH | tsp.DEV_BAD_PAGE
    assert np.array_equal(f64(pools[1]), ref[2])
    for x, r in ((out, ref[0]), (pools[0], ref[1])):
        assert (np.abs(f64(x) - r) <= HALF_STEP * (np.abs(r) + 2.0 ** -17) + 2.0 ** -17).all()


# ---------------------------------------------------------------- attention

def attend(rng, B, T, Hq, Hkv, D, ps, lens, causal, layout=lambda x: x, scale=0.0, sharp=1.0):
    """Runs a call on a pool whose unused rows are NaN and compares it; returns the device tensors."""
    cap = max(1, -(-max(lens) // ps))
    table, pages = make_table(rng, B, cap)
    kp, vp = normal(rng, pages, ps, Hkv, D), normal(rng, pages, ps, Hkv, D)
    q = bf16_round(sharp * rng.standard_normal((B, T, Hq, D)))
    used = np.zeros((pages, ps), bool)
    for b, n in enumerate(lens):
        s = np.arange(n)
        used[table[b, s // ps], s % ps] = True
        table[b, -(-n // ps):] = -1
    kp[~used], vp[~used] = np.nan, np.nan
    ref, weight = oracle.paged_attention(q, kp, vp, table, lens, causal, scale or None)
    t = (bf(q), layout(bf(kp)), layout(bf(vp)), i32(table), i32(lens))
    out = tsp.paged_attn(*t, causal=causal, scale=scale)
    assert tsp.device_status() == 0
    err = np.abs(f64(out) - ref)
    tol = (HALF_STEP + 2.0 ** -10) * weight + HALF_STEP * np.abs(ref) + 1e-30
    assert (err <= tol).all(), float((err - tol).max())
    return t, out


ATTEND = [
    # T, Hq, Hkv, D, page_size, lens
    (1, 4, 4, 64, 16, [192]),
    (1, 2, 2, 128, 32, [0, 1, 31, 32, 33, 127, 128, 129, 300]),
    (1, 16, 1, 64, 64, [1000, 77, 0, 5]),
    (1, 17, 1, 128, 16, [100, 260]),                  # 17 rows: a second fragment of one row
    (3, 14, 2, 128, 24, [500, 2, 3, 0, 129]),          # causal: rows before the sequence's start see nothing
    (5, 4, 4, 64, 5, [777, 4, 131]),
    (32, 4, 1, 128, 1, [200, 33]),                     # four row tiles
    (64, 2, 2, 64, 736, [736, 64, 65, 100]),
    (33, 1, 1, 128, 48, [400]),
    (2, 8, 2, 64, 100, [4000, 1]),                     # one long sequence: split over many workgroups
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,ps,lens", ATTEND)
def test_attention_parity(T, Hq, Hkv, D, ps, lens, causal):
    attend(np.random.default_rng(T + ps), len(lens), T, Hq, Hkv, D, ps, lens, causal)


PADDED = [
    # T, Hq, Hkv, D, page_size, cached before, n_new: each kernel, in one range and in several
    (7, 4, 2, 128, 16, [0, 20, 33, 0], [7, 0, 3, 1]),
    (7, 4, 2, 64, 5, [4000, 20, 133, 2], [7, 0, 3, 6]),
    (13, 4, 2, 128, 32, [3000, 0], [13, 4]),
    (32, 2, 1, 128, 16, [100, 2500, 0], [0, 17, 32]),
    (70, 8, 2, 64, 48, [0, 1200, 31], [69, 70, 1]),
    (70, 8, 2, 128, 20, [5, 0], [33, 2]),
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,ps,before,n_new", PADDED)
def test_appended_and_attended_in_a_padded_batch(T, Hq, Hkv, D, ps, before, n_new, causal):
    """Padding is NaN in q, k and v, and pages behind a sequence's last token are not in the table."""
    rng = np.random.default_rng(T + Hq + ps)
    B = len(before)
    lens = np.add(before, n_new)
    table, pages = make_table(rng, B, -(-int(lens.max()) // ps))
    kp, vp = np.full((pages, ps, Hkv, D), np.nan), np.full((pages, ps, Hkv, D), np.nan)
    for b in range(B):
        s = np.arange(before[b])
        kp[table[b, s // ps], s % ps], vp[table[b, s // ps], s % ps] = normal(rng, before[b], Hkv, D), normal(rng, before[b], Hkv, D)
        table[b, -(-lens[b] // ps):] = -1
    q, k, v = normal(rng, B, T, Hq, D), normal(rng, B, T, Hkv, D), normal(rng, B, T, Hkv, D)
    for b in range(B):
        for x in (q, k, v):
            x[b, n_new[b]:] = np.nan
    pools, new = (bf(kp), bf(vp)), i32(n_new)
    tsp.paged_append(bf(k), bf(v), *pools, i32(table), i32(before), n_new=new, rope_theta=0.0)
    _, kp, vp = oracle.paged_append(None, k, v, kp, vp, table, before, n_new, theta=0)
    ref, weight = oracle.paged_attention(q, kp, vp, table, lens, causal, n_new=n_new)
    out = f64(tsp.paged_attn(bf(q), *pools, i32(table), i32(lens), causal=causal, n_new=new))
    assert tsp.device_status() == 0
    assert (np.abs(out - ref) <= (HALF_STEP + 2.0 ** -10) * weight + HALF_STEP * np.abs(ref) + 1e-30).all()
    for b in range(B):
        assert (out[b, n_new[b]:] == 0).all()


def test_attention_clamps_the_number_of_new_tokens():
    rng = np.random.default_rng(12)
    t, _ = attend(rng, 3, 4, 2, 1, 64, 16, [30, 300, 9], True)
    out = tsp.paged_attn(*t, causal=True, n_new=i32([5, 4, -1]))
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH
    assert torch.equal(out, tsp.paged_attn(*t, causal=True, n_new=i32([4, 4, 0]))) and tsp.device_status() == 0


def test_attention_over_pages_of_heads_and_other_scales():
    rng = np.random.default_rng(8)
    for layout, ps in ((heads_first, 16), (heads_first, 20)):
        attend(rng, 3, 2, 8, 4, 128, ps, [90, 400, 1], True, layout=layout, scale=0.3)
    attend(rng, 2, 1, 4, 2, 64, 16, [1500, 40], False, sharp=8.0)  # peaked weights: the maximum moves often


def test_attention_of_many_sequences():
    """More sequences than a wave has lanes, lengths from nothing to long."""
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 90, 150)
    lens[[3, 64, 149]] = 3000, 0, 1111
    attend(rng, 150, 1, 2, 1, 64, 16, lens.tolist(), False)


def test_attention_unsplit_and_in_a_larger_workspace_agree():
    rng = np.random.default_rng(10)
    t, out = attend(rng, 2, 2, 8, 2, 128, 32, [3000, 700], False)
    lib = tsp.load()
    import ctypes
    from paper_2608_27514_amd import _lib
    q, kp, vp, table, lens = t
    sh = _lib._paged_struct(*_lib._paged_sizes(2, 2, 8, kp, vp, table, 0))[0]
    whole = torch.empty_like(q)
    ptr = [x.data_ptr() for x in (q, kp, vp, table, lens)] + [None, whole.data_ptr()]
    assert lib.traj_paged_attn(*ptr, ctypes.byref(sh), 0.0, 0, None, 0, torch.cuda.current_stream().cuda_stream) == 0
    # both within half a step of the weights' rounding (of values near 1: some 2^-7) and of their own
    assert (whole.float() - out.float()).abs().max().item() <= 2.0 ** -6
    need = tsp.paged_attn_workspace_size(q, kp, vp, table)
    assert need > 0
    big = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")  # NaN in every float
    assert torch.equal(tsp.paged_attn(*t, workspace=big), out)
    assert (big[need:] == 255).all()


def test_attention_bad_lengths_and_pages():
    rng = np.random.default_rng(11)
    B, T, H, D, ps = 3, 1, 2, 64, 16
    table = np.array([[0, 1], [2, 77], [-1, 3]], np.int32)
    kp, vp, q = normal(rng, 4, ps, H, D), normal(rng, 4, ps, H, D), normal(rng, B, T, H, D)
    lens = [1000, 30, 20]
    for page in (ps, 8):  # the same pool in pages within a tile's blocks, and smaller ones
        k8, v8 = kp.reshape(-1, page, H, D), vp.reshape(-1, page, H, D)
        f = ps // page
        t8 = np.where((table >= 0) & (table < 4), table, -99)[:, :, None] * f + np.arange(f) if f > 1 else table[:, :, None]
        t8 = t8.reshape(B, -1).astype(np.int32)
        ref, weight = oracle.paged_attention(q, k8, v8, t8, lens)
        tsp.device_status()
        out = tsp.paged_attn(bf(q), bf(k8), bf(v8), i32(t8), i32(lens))
        assert tsp.device_status() == tsp.DEV_BAD_LENGTH | tsp.DEV_BAD_PAGE
        assert (np.abs(f64(out) - ref) <= (HALF_STEP + 2.0 ** -10) * weight + HALF_STEP * np.abs(ref) + 1e-30).all()
    out = tsp.paged_attn(bf(q), bf(kp), bf(vp), i32(table), i32([-5, 0, -1]))
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH
    assert not out.any()


def test_offsets_past_32_bits():
    """A pool of more than 2^32 values: its last pages are written and read."""
    rng = np.random.default_rng(12)
    ps, Hkv, D, T = 64, 8, 128, 3
    pages = (2 ** 32 + 2 ** 27) // (ps * Hkv * D)
    kp = torch.empty(pages, ps, Hkv, D, dtype=BF, device="cuda")
    vp = torch.empty_like(kp)
    table = np.array([[pages - 1, pages - 3, 0]], np.int32)
    n = 2 * ps + 10
    k, v, q = normal(rng, 1, n, Hkv, D), normal(rng, 1, n, Hkv, D), normal(rng, 1, T, Hkv, D)
    tsp.paged_append(bf(k), bf(v), kp, vp, i32(table), i32([0]), rope_theta=0.0)
    out = tsp.paged_attn(bf(q), kp, vp, i32(table), i32([n]))
    small = np.arange(3, dtype=np.int32)[None]
    pad = ((0, 3 * ps - n), (0, 0), (0, 0))
    ref, weight = oracle.paged_attention(q, np.pad(k[0], pad).reshape(3, ps, Hkv, D), np.pad(v[0], pad).reshape(3, ps, Hkv, D), small, [n])
    assert (np.abs(f64(out) - ref) <= (HALF_STEP + 2.0 ** -10) * weight + HALF_STEP * np.abs(ref)).all()
    assert torch.equal(kp[pages - 1].cpu(), bf(k)[0, :ps].cpu())


def test_empty_batches_do_nothing():
    kp = torch.zeros(2, 16, 2, 64, dtype=BF, device="cuda")
    for B, T in ((0, 3), (2, 0)):
        x = torch.zeros(B, T, 2, 64, dtype=BF, device="cuda")
        table, n = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        assert tsp.paged_append(x, x, kp, kp.clone(), table, n, q=x).shape == x.shape
        assert tsp.paged_attn(x, kp, kp, table, n).shape == x.shape


def test_append_then_attend_matches_verification_over_a_contiguous_cache():
    """A denoising step's block written to the cache and attended to: what verify_attn computes for one draft whose
    keys are its own block."""
    rng = np.random.default_rng(13)
    L, H, D, S = 32, 4, 128, 200
    q, k, v = (bf(normal(rng, 1, 1, L, H, D)) for _ in range(3))
    kc, vc = bf(normal(rng, 1, S, H, D)), bf(normal(rng, 1, S, H, D))
    want = tsp.verify_attn(q, kc, vc, k, v, i32([[-1]]))
    ps = 16
    pages = -(-(S + L) // ps)
    pools = [torch.zeros(pages, ps, H, D, dtype=BF, device="cuda") for _ in range(2)]
    table = i32(rng.permutation(pages)[None])
    tsp.paged_append(kc, vc, *pools, table, i32([0]), rope_theta=0.0)
    tsp.paged_append(k[0], v[0], *pools, table, i32([S]), rope_theta=0.0)
    got = tsp.paged_attn(q[0], *pools, table, i32([S + L]))
    # each is within 2^-8 of the weights' rounding, with values near 1 / sqrt(keys), and half a step of the other
    assert (got.float() - want[0].float()).abs().max().item() <= 2.0 ** -8
