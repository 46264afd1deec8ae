"""GPU parity: confidences of adjusted logits against the oracle.  The adjusted values are the same fp32 operations on
both sides, so candidates are equal; confidences within 1e-4 (fp32 exponentials and sums)."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import CONF_ATOL, cuda
from oracle.layer import bf16_round

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def make(rng, seqs, per, V, H=0, NB=0, masks=0, density=0.5, dtype=BF):
    """numpy inputs of a call, with repeated tokens, padding, duplicate biases and a planted token per row."""
    R = seqs * per
    x = rng.standard_normal((R, V)).astype(np.float32)
    x[np.arange(R), rng.integers(0, V, R)] += np.log(V) + 2
    if dtype == BF:
        x = bf16_round(x).astype(np.float32)
    how = {}
    if H:
        how["history"] = rng.integers(-2, V + 2, (seqs, H)).astype(np.int32)
        how["history"][:, ::2] = rng.integers(0, min(V, 7), (seqs, (H + 1) // 2))
        how["history"][:, -1] = x[::per].argmax(1)
        how["history_len"] = rng.integers(0, H + 1, seqs).astype(np.int32)
        how["history_len"][0] = H
        how["repetition"] = rng.uniform(0.7, 2, seqs).astype(np.float32)
        how["frequency"] = rng.uniform(-0.2, 0.5, seqs).astype(np.float32)
        how["presence"] = rng.uniform(-0.2, 0.5, seqs).astype(np.float32)
    if NB:
        how["bias_ids"] = rng.integers(-1, V + 1, (seqs, NB)).astype(np.int32)
        how["bias"] = (3 * rng.standard_normal((seqs, NB))).astype(np.float32)
        how["bias"][:, 0] = -np.inf
        if NB > 2:
            how["bias_ids"][:, 2] = how["bias_ids"][:, 1]  # the same token twice
    if masks:
        how["mask"] = np.packbits(rng.random((masks, -(-V // 32) * 32)) < density, axis=1, bitorder="little").view(np.uint32)
        how["mask_index"] = rng.integers(-1, masks, R).astype(np.int32)
    return x, how


def on_gpu(x, how, dtype):
    up = {n: cuda(v.view(np.int32) if v.dtype == np.uint32 else v) for n, v in how.items()}
    return cuda(x, dtype), up


def check(x, how, k, per, dtype=BF, logits=None):
    lg, up = on_gpu(x, how, dtype)
    conf, idx = tsp.confidence_topk_adjusted(lg if logits is None else logits, k, per, **up)
    torch.cuda.synchronize()
    rc, ri = oracle.confidence_topk_adjusted(x, k, per, **how)
    assert np.array_equal(idx.cpu().numpy(), ri)
    assert np.abs(conf.cpu().numpy() - rc).max() <= CONF_ATOL
    assert (conf.cpu().numpy()[ri < 0] == 0).all()
    return conf, idx


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("seqs,per,V,H,NB,masks,density,k", [
    (1, 1, 126464, 500, 4, 0, 0, 3),          # one row: split over workgroups
    (2, 8, 50257, 33, 300, 0, 0, 5),          # rows start at any element
    (3, 5, 1000, 64, 0, 4, 0.3, 8),
    (1, 40, 8, 3, 2, 3, 0.5, 8),              # a vocabulary smaller than a vector
    (2, 2, 33, 0, 0, 2, 0.1, 4),
    (2, 3, 4099, 5000, 1, 1, 0.9, 2),         # more records than are counted at a time
    (4, 1, 32000, 1, 1, 4, 0.002, 3),         # narrow masks
    (130, 2, 3001, 10, 3, 9, 0.5, 1),
    (3, 200, 2048, 20, 5, 60, 0.02, 4),
])
def test_parity(seqs, per, V, H, NB, masks, density, k, dtype):
    x, how = make(np.random.default_rng(V + k), seqs, per, V, H, NB, masks, density, dtype)
    check(x, how, min(k, V), per, dtype)
    assert tsp.device_status() == 0


def test_each_part_alone_and_none():
    rng = np.random.default_rng(5)
    x, how = make(rng, 3, 4, 5000, 50, 6, 5, 0.2)
    for names in ((), ("history",), ("history", "repetition"), ("history", "frequency", "history_len"), ("history", "presence"),
                  ("bias_ids", "bias"), ("mask", "mask_index")):
        check(x, {n: how[n] for n in names}, 3, 4)
    lg, _ = on_gpu(x, {}, BF)
    conf, idx = tsp.confidence_topk_adjusted(lg, 3, 4)
    conf0, idx0 = tsp.confidence_topk(lg, 3)
    assert torch.equal(idx, idx0)
    assert (conf - conf0).abs().max().item() <= 2 * CONF_ATOL  # each is within CONF_ATOL of the same value


def test_a_mask_per_row_and_a_strided_one():
    rng = np.random.default_rng(6)
    x, how = make(rng, 2, 3, 700, masks=6, density=0.3)
    how["mask"] = np.concatenate([how["mask"], np.full((6, 3), 0xFFFFFFFF, np.uint32)], 1)
    del how["mask_index"]
    check(x, how, 3, 3)


def test_rows_of_a_wider_matrix_and_the_last_row_ragged():
    rng = np.random.default_rng(7)
    for dtype in (BF, F32):
        x, how = make(rng, 3, 4, 1237, 20, 4, 3, 0.4, dtype)
        x = x[:9]  # the third sequence has one row
        how["mask_index"] = how["mask_index"][:9]
        wide = torch.full((9, 1301), float("nan"), dtype=dtype, device="cuda")
        wide[:, 5:5 + 1237] = cuda(x, dtype)
        check(x, how, 4, 4, dtype, logits=wide[:, 5:5 + 1237])


def test_rows_that_allow_few_tokens_or_none():
    V, k = 4000, 4
    rng = np.random.default_rng(8)
    x, _ = make(rng, 1, 6, V)
    mask = np.zeros((5, V // 32), np.uint32)
    mask[1, 17] = 1 << 5
    mask[2, [0, 124]] = 1, 1 << 31
    mask[3] = 0xFFFFFFFF
    how = dict(mask=mask, mask_index=np.array([0, 1, 2, 3, 4, -1], np.int32))
    # what is forbidden may hold anything
    free = oracle.adjust_logits(np.zeros_like(x), 6, **how) == 0
    x[~free] = np.where(rng.random((~free).sum()) < 0.5, np.nan, np.inf)
    conf, idx = check(x, how, k, 6)
    assert idx[0].tolist() == [-1] * 4 and idx[1].tolist() == [17 * 32 + 5, -1, -1, -1] and conf[1, 0] == 1
    # everything banned by bias or by the model itself
    x = np.full((2, 64), -np.inf, np.float32)
    check(x, {}, 3, 1)
    x[:, 7] = 2.0
    how = dict(bias_ids=np.array([[7], [7]], np.int32), bias=np.array([[-np.inf], [1.0]], np.float32))
    check(x, how, 3, 1)


def test_values_at_the_ends_of_their_range():
    """Logits at the type's lowest and far apart, and ties: the lower index first."""
    x = np.zeros((3, 300), np.float32)
    x[0] = torch.finfo(BF).min
    x[0, 200:204] = -5.0
    x[1] = -60.0
    x[1, [9, 80]] = 60.0
    x[2, ::7] = 1.5
    history = np.array([[200, 201, 201], [9, 9, 9], [0, 7, -1]], np.int32)
    how = dict(history=history, repetition=np.array([2, 2, 2], np.float32), frequency=np.array([1, 0, 0], np.float32))
    check(x, how, 5, 1)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_of_the_lowest_and_of_huge_values(dtype):
    """Logits masked by the type's lowest value, rows of nothing else, and ones that a product with log2(e) overflows."""
    big = float(torch.finfo(dtype).max)
    V = 5003
    x = np.full((7, V), -big, np.float32)
    x[0, 77] = 1.0
    x[1, :4000] = -1e30
    x[2, 3:6] = big
    x[3] = 0.0
    x[3, 4999] = big
    x[4] = bf16_round(2000 + np.arange(V) % 13)
    x[5, 1000] = -1e38
    how = dict(history=np.array([[77, 5], [9, 9], [3, 1], [0, 7], [1, 1], [2, 1000], [5, 6]], np.int32), repetition=np.full(7, 1.5, np.float32))
    check(x, {}, 4, 1, dtype)
    check(x, how, 4, 1, dtype) if dtype == BF else check(np.clip(x, -2e38, 2e38), how, 4, 1, dtype)


def test_many_history_tokens_and_duplicates():
    """Every token of the vocabulary in the history, and one token many times."""
    V = 6000
    rng = np.random.default_rng(9)
    x, _ = make(rng, 2, 1, V)
    h = np.stack([rng.permutation(np.repeat(np.arange(V), 2)), np.full(2 * V, 11)]).astype(np.int32)
    how = dict(history=h, repetition=np.array([1.3, 1.2], np.float32), frequency=np.array([0.25, 0.001], np.float32),
               presence=np.array([0.5, 0.1], np.float32))
    check(x, how, 8, 1)
    how = dict(bias_ids=np.full((2, 40), 4321, np.int32), bias=rng.standard_normal((2, 40)).astype(np.float32))
    check(x, how, 3, 1)


def test_a_list_padded_with_one_token():
    """Some tokens are named once, some a few times and one in most of the list, as padding of a real token with 0 would."""
    V, NB = 4099, 1500
    rng = np.random.default_rng(12)
    x, _ = make(rng, 3, 2, V)
    ids = rng.integers(0, V, (3, NB)).astype(np.int32)
    bias = rng.standard_normal((3, NB)).astype(np.float32)
    ids[0, 100:], bias[0, 100:] = 0, 0
    ids[1, ::2] = 17
    ids[2, 200:] = np.tile(rng.permutation(V)[:130], 10)
    check(x, dict(bias_ids=ids, bias=bias), 8, 2)
    h = rng.integers(0, V, (3, 40)).astype(np.int32)
    check(x, dict(bias_ids=ids, bias=bias, history=h, presence=np.full(3, 0.5, np.float32)), 4, 2)


def test_largest_vocabulary():
    V = 1 << 19
    rng = np.random.default_rng(10)
    x, how = make(rng, 1, 2, V, 100, 5, 2, 0.7)
    check(x, how, 3, 2)


def test_bad_indices_are_reported():
    rng = np.random.default_rng(11)
    x, how = make(rng, 2, 2, 500, 10, 0, 3, 0.5)
    how["mask_index"] = np.array([0, 3, -2, -1], np.int32)
    how["history_len"] = np.array([-1, 11], np.int32)
    tsp.device_status()
    check(x, how, 3, 2)
    assert tsp.device_status() == tsp.DEV_BAD_MASK | tsp.DEV_BAD_HISTORY


def test_workspaces():
    rng = np.random.default_rng(12)
    x, how = make(rng, 2, 3, 40000, 50, 4, 2, 0.5)
    lg, up = on_gpu(x, how, BF)
    need = tsp.confidence_topk_adjusted_workspace_size(lg, 3, 3, history=up["history"], bias=up["bias"])
    want = tsp.confidence_topk_adjusted(lg, 3, 3, **up)
    ws = torch.full((need + 1024,), 255, dtype=torch.uint8, device="cuda")
    for a, b in zip(tsp.confidence_topk_adjusted(lg, 3, 3, workspace=ws, **up), want):
        assert torch.equal(a, b)
    assert (ws[need:] == 255).all()
    with pytest.raises(tsp.TrajSpecError, match="E_WORKSPACE"):
        tsp.confidence_topk_adjusted(lg, 3, 3, workspace=ws[:1024], **up)


def test_no_rows():
    x = torch.zeros(0, 100, dtype=BF, device="cuda")
    conf, idx = tsp.confidence_topk_adjusted(x, 3, 4, mask=torch.zeros(1, 4, dtype=torch.int32, device="cuda"),
                                             mask_index=torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert conf.shape == idx.shape == (0, 3)
