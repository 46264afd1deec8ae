"""Appends to an 8-bit cache in front of tokens that stay: a block that is denoised before a cached suffix.  Values match the
oracle bit for bit; keys that are rotated as in the appends' other tests."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import cuda
from oracle import eight
from oracle.layer import bf16_round
from test_gpu_eight import E4, bf, bytes_of, check_append, f64, heads_first, i32, make_pools, make_table, normal, on_gpu

pytestmark = pytest.mark.gpu


def same(got, pools):
    return all(np.array_equal(f64(x) if x.dtype == E4 else bytes_of(x), want) for x, want in zip(got, pools))


@pytest.mark.parametrize("D,ps,sb", [(128, 16, 16), (64, 24, 8), (128, 64, 64), (64, 48, 24), (128, 32, 1), (128, 60, 5), (64, 64, 32)])
def test_from_every_offset_to_every_length(D, ps, sb):
    """A sequence for each place of a page to begin at; lengths before, in and behind the call's last block."""
    rng = np.random.default_rng(D + ps + sb)
    for T in (1, 7, 16, 17, 33, 70):
        columns = -(-(2 * ps + T) // ps)
        table, pages = make_table(rng, ps, columns)
        before = make_pools(rng, pages, ps, sb, 2, D)
        k, v = (bf16_round(rng.standard_normal((ps, T, 2, D)) * 2.0 ** rng.integers(-3, 4, (ps, T, 1, 1))) for _ in range(2))
        start, n_new = np.arange(ps, dtype=np.int32), rng.integers(0, T + 1, ps).astype(np.int32)
        lens = np.maximum(start + n_new + rng.integers(-2, sb + 3, ps), 0).astype(np.int32)
        lens[:2] = columns * ps, 0
        _, pools, _ = eight.paged_append8(k, k, v, before, table, start, n_new, theta=0, lens=lens)
        got = on_gpu(before, heads_first if T % 2 else lambda x: x)
        tsp.paged_append8(bf(k), bf(v), *got, i32(table), i32(start), n_new=i32(n_new), rope_theta=0.0, lens=i32(lens))
        assert tsp.device_status() == 0
        assert same(got, pools), T
        # nothing of the sequence behind a call: the same as without lengths
        _, pools, _ = eight.paged_append8(k, k, v, before, table, start, n_new, theta=0)
        got = on_gpu(before)
        tsp.paged_append8(bf(k), bf(v), *got, i32(table), i32(start), n_new=i32(n_new), rope_theta=0.0, lens=i32(start + n_new))
        assert tsp.device_status() == 0 and same(got, pools), T


def test_rotated_keys_and_queries():
    rng = np.random.default_rng(1)
    B, T, Hq, Hkv, D, ps, sb = 5, 40, 8, 2, 128, 48, 24
    start, n_new, lens, pos0 = [0, 17, 47, 48, 100], [40, 39, 1, 20, 0], [200, 60, 49, 71, 130], [5, 6, 7, 1000, 1]
    qkv = bf16_round(rng.standard_normal((B, T, (Hq + 2 * Hkv) * D)) * 2.0 ** rng.integers(-3, 4, (B, T, 1)))
    table, pages = make_table(rng, B, 5)
    before = make_pools(rng, pages, ps, sb, Hkv, D)
    q, k, v = (x.reshape(B, T, -1, D) for x in np.split(qkv, [Hq * D, (Hq + Hkv) * D], axis=-1))
    ref, pools, exact = eight.paged_append8(q, k, v, before, table, start, n_new, pos0, lens=lens)
    size = eight.paged_append8(np.abs(q) + np.abs(np.roll(q, D // 2, -1)), k, v, before, table, start, n_new, pos0, 0)[0]
    qg, kg, vg = (x.view(B, T, -1, D) for x in bf(qkv).split([Hq * D, Hkv * D, Hkv * D], -1))
    got = on_gpu(before)
    out = tsp.paged_append8(kg, vg, *got, i32(table), i32(start), q=qg, n_new=i32(n_new), pos0=i32(pos0), lens=i32(lens))
    assert tsp.device_status() == 0
    check_append(got, out, (ref, size), pools, exact, qkv, 500000.0)


def test_a_block_denoised_in_front_of_a_suffix():
    """Steps that write a block in the middle of the sequences and attend to all of them: the suffix keeps its values, whatever
    the block's borders, and one whose borders are those of scale blocks keeps its bits and scales without any lengths."""
    rng = np.random.default_rng(2)
    B, T, Hq, Hkv, D, ps, sb = 3, 32, 4, 2, 64, 32, 16
    table, pages = make_table(rng, B, 5)
    pools = make_pools(rng, pages, ps, sb, Hkv, D)
    lens = np.array([150, 101, 160], np.int32)
    for start in ([37, 60, 80], [64, 32, 112]):
        aligned = start[0] == 64
        prompt = [bf16_round(rng.standard_normal((B, 160, Hkv, D)) * 2.0 ** rng.integers(-2, 3, (B, 160, 1, 1))) for _ in range(2)]
        _, pools, _ = eight.paged_append8(None, *prompt, pools, table, [0] * B, lens, theta=0)
        got = on_gpu(pools)
        first = [eight.paged_values(pools[i], pools[2 + i]) for i in (0, 1)]
        t, s, n = i32(table), i32(start), i32(lens)
        for step in range(3):
            q, k, v = (normal(rng, B, T, h, D) * 2.0 ** (step * (h == Hkv)) for h in (Hq, Hkv, Hkv))
            _, pools, _ = eight.paged_append8(None, k, v, pools, table, start, theta=0, lens=None if aligned else lens)
            tsp.paged_append8(bf(k), bf(v), *got, t, s, rope_theta=0.0, lens=None if aligned else n)
            assert same(got, pools), step
            kp, vp = (eight.paged_values(pools[i], pools[2 + i]) for i in (0, 1))
            ref, weight = oracle.paged_attention(q, kp, vp, table, lens)
            out = tsp.paged_attn8(bf(q), *got, t, n)
            assert tsp.device_status() == 0
            assert (np.abs(f64(out) - ref) <= 2.0 ** -10 * weight + 2.0 ** -8 * np.abs(ref)).all()
        for b in range(B):
            for at in [*range(start[b]), *range(start[b] + T, lens[b])]:
                page, row = table[b, at // ps], at % ps
                for i, x in enumerate((kp, vp)):
                    # each growth of a scale may cost half a step of 2^-9 of it; three steps, scales that double: under twice the last
                    tol = 0.0 if aligned else 2 * 2.0 ** -10 * eight.scale_value(pools[2 + i][page, row // sb])[:, None]
                    assert (np.abs(x[page, row] - first[i][page, row]) <= tol).all(), (b, at)


def test_bad_lengths_and_pages():
    rng = np.random.default_rng(3)
    H, D, ps, sb, T = 1, 64, 8, 8, 3
    table = np.array([[0, 1], [2, 99], [3, 4], [-1, 5]], np.int32)
    before = make_pools(rng, 6, ps, sb, H, D)
    k, v = (bf16_round(8 * rng.standard_normal((4, T, H, D))) for _ in range(2))
    start = [2, 9, 14, 1]
    for lens in ([8, 16, 16, 8], [1000, -1, 17, 7]):
        _, pools, _ = eight.paged_append8(None, k, v, before, table, start, theta=0, lens=lens)
        got = on_gpu(before)
        tsp.device_status()
        tsp.paged_append8(bf(k), bf(v), *got, i32(table), i32(start), rope_theta=0.0, lens=i32(lens))
        assert tsp.device_status() == tsp.DEV_BAD_PAGE | tsp.DEV_BAD_LENGTH  # start[2] + 3 > 16, pages 99 and -1
        assert same(got, pools)
    got = on_gpu(before)
    tsp.paged_append8(bf(k[:1]), bf(v[:1]), *got, i32(table[:1]), i32([2]), rope_theta=0.0, lens=i32([17]))
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH


def test_captured_and_replayed():
    """Lengths are read at each replay."""
    rng = np.random.default_rng(4)
    B, T, H, D, ps, sb = 2, 5, 2, 128, 16, 16
    table, pages = make_table(rng, B, 3)
    pools = make_pools(rng, pages, ps, sb, H, D)
    got, t = on_gpu(pools), i32(table)
    k, v, s, n = bf(np.zeros((B, T, H, D))), bf(np.zeros((B, T, H, D))), i32([0, 0]), i32([0, 0])
    tsp.paged_append8(k, v, *on_gpu(pools), t, s, rope_theta=0.0, lens=n)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tsp.paged_append8(k, v, *got, t, s, rope_theta=0.0, lens=n)
    for start, lens in (([3, 20], [16, 30]), ([0, 11], [5, 48]), ([30, 16], [34, 32])):
        x = bf16_round(rng.standard_normal((2, B, T, H, D)) * 4)
        k.copy_(bf(x[0]))
        v.copy_(bf(x[1]))
        s.copy_(i32(start))
        n.copy_(i32(lens))
        graph.replay()
        _, pools, _ = eight.paged_append8(None, *x, pools, table, start, theta=0, lens=lens)
        torch.cuda.synchronize()
        assert same(got, pools)


def test_the_binding_refuses():
    x, kp = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 16, 2, 64, dtype=E4, device="cuda")
    scale = torch.full((4, 1, 2), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    table, n = cuda(np.arange(4, dtype=np.int32).reshape(2, 2)), cuda(np.zeros(2, np.int32))
    for bad in (n.long(), n[:1], n.cpu()):
        with pytest.raises((TypeError, ValueError)):
            tsp.paged_append8(x, x, kp, kp.clone(), scale, scale.clone(), table, n, lens=bad)


def test_calls_that_begin_before_the_cache_or_end_at_its_end():
    """Tokens without a place lie in blocks of their own; the last block of the table may be the call's last, or full."""
    rng = np.random.default_rng(5)
    H, D, ps, sb, T = 2, 64, 16, 8, 6
    table, pages = make_table(rng, 4, 2)
    before = make_pools(rng, pages, ps, sb, H, D)
    before[2][:] = rng.integers(0, 256, before[2].shape)  # bytes outside [27, 247] count as the nearest
    k, v = (bf16_round(rng.standard_normal((4, T, H, D)) * 2.0 ** rng.integers(-3, 8, (4, T, 1, 1))) for _ in range(2))
    start, n_new, lens = [-3, 24, 26, 25], [6, 5, 6, 0], [32, 32, 32, 32]
    _, pools, _ = eight.paged_append8(k, k, v, before, table, start, n_new, theta=0, lens=lens)
    got = on_gpu(before)
    tsp.device_status()
    tsp.paged_append8(bf(k), bf(v), *got, i32(table), i32(start), n_new=i32(n_new), rope_theta=0.0, lens=i32(lens))
    assert tsp.device_status() == tsp.DEV_BAD_LENGTH and same(got, pools)
