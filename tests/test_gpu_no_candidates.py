"""Rows that allow fewer than k tokens (idx -1, confidence 0), through the calls that take candidates: parity with the
oracles, on tables of such rows and behind the adjusted logit pass."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import cuda
from oracle.tree import build_tree_batch

pytestmark = pytest.mark.gpu
I32, F32 = torch.int32, torch.float32


def table(rng, shape, k, most):
    """Candidates of rows that allow 0 to `most` tokens."""
    allowed = rng.integers(0, most + 1, shape)
    conf = np.sort(rng.random(shape + (k,)), -1)[..., ::-1].astype(np.float32)
    idx = (np.argsort(rng.random(shape + (64,)), axis=-1)[..., :k] + 100).astype(np.int32)
    none = np.arange(k) >= allowed[..., None]
    conf[none], idx[none] = 0, -1
    return conf, idx


def check_tree(out, ref):
    t, p, n, s = ref
    assert np.array_equal(out["n_nodes"].cpu().numpy(), n)
    assert np.array_equal(out["parent"].cpu().numpy(), p)
    assert np.array_equal(out["tokens"].cpu().numpy(), t)
    got, fin = out["score"].cpu().numpy(), np.isfinite(s)
    assert np.array_equal(np.isfinite(got), fin)
    assert (np.abs(got[fin] - s[fin]) <= 1e-5 * (1 + np.abs(s[fin]))).all()  # fp32 sums of logf


@pytest.mark.parametrize("seed", range(24))
def test_trees_of_rows_with_few_tokens(seed):
    rng = np.random.default_rng(seed)
    B, L, k = int(rng.integers(1, 30)), int(rng.choice([1, 2, 7, 32, 64])), int(rng.integers(1, 9))
    W, D = int(rng.integers(1, 5)), int(rng.integers(0, 6))
    branch, deep, full = int(rng.integers(1, k + 1)), int(rng.integers(1, k + 1)), bool(seed % 2)
    tau = float(np.float32(rng.choice([0.3, 0.9, 0.95])))
    if tsp.tree_max_nodes(B, L, k, W, D, branch, full, deep) > 64:
        deep = 1
    state = np.where(rng.random((B, L)) < 0.8, -1, rng.integers(0, 1000, (B, L))).astype(np.int32)
    most = (0, 1, 2, k)[seed % 4]
    conf, idx = table(rng, (B, L), k, most)
    n_max = tsp.tree_max_nodes(B, L, k, W, D, branch, full, deep)
    out = tsp.build_tree(cuda(state), cuda(conf), cuda(idx), tau, W, D, branch, full, branch_deep=deep)
    check_tree(out, build_tree_batch(state, None, None, None, conf, idx, tau, W, D, branch, full, n_max, deep))
    n, parent, tokens = (out[m].cpu().numpy() for m in ("n_nodes", "parent", "tokens"))
    for b in range(B):  # no node equals what it was generated from
        for i in range(n[b]):
            assert not np.array_equal(tokens[b, i], state[b] if parent[b, i] < 0 else tokens[b, parent[b, i]])


def adjusted_candidates(rng, B, L, k, V):
    """Candidates of a step under masks of 0 to 5 tokens, as the logit pass gives them and as its oracle does."""
    logits = (2 * rng.standard_normal((B * L, V))).astype(np.float32)
    bits = np.zeros((7, V), np.uint8)
    for m in range(6):
        bits[m, rng.choice(V, m, replace=False)] = 1
    bits[6] = 1
    mask = np.packbits(np.pad(bits, ((0, 0), (0, -V % 32))), axis=1, bitorder="little").view(np.uint32)
    index = rng.integers(0, 7, B * L).astype(np.int32)
    index[:L] = 0  # the first sequence allows nothing at all
    conf, idx = tsp.confidence_topk_adjusted(cuda(logits), k, L, mask=cuda(mask.view(np.int32)), mask_index=cuda(index))
    ri = oracle.confidence_topk_adjusted(logits, k, L, mask=mask, mask_index=index)[1]
    assert np.array_equal(idx.cpu().numpy(), ri) and (ri[:L] == -1).all() and (ri >= 0).any()
    return conf.view(B, L, k), idx.view(B, L, k)


def test_a_tree_behind_adjusted_logits():
    rng = np.random.default_rng(1)
    B, L, k, tau = 5, 16, 3, float(np.float32(0.6))
    conf, idx = adjusted_candidates(rng, B, L, k, 500)
    state = np.full((B, L), -1, np.int32)
    out = tsp.build_tree(cuda(state), conf, idx, tau, 3, 3, 3)
    c, i = conf.cpu().numpy(), idx.cpu().numpy()
    check_tree(out, build_tree_batch(state, None, None, None, c, i, tau, 3, 3, 3, False, out["parent"].shape[1]))
    assert out["n_nodes"][0] == 0 and (out["tokens"][0] == -1).all()
    assert torch.equal(out["conf_next"], conf) and torch.equal(out["idx_next"], idx)


def check_accept(out, ref):
    for name in ("leaf", "n_accepted", "out_tokens", "on_path", "hi"):
        got = out[name].cpu().numpy()
        assert np.array_equal(got.astype(bool) if ref[name].dtype == bool else got, ref[name]), name


@pytest.mark.parametrize("traversal", ["greedy", "longest"])
@pytest.mark.parametrize("mode", ["exact", "top1", "topk"])
@pytest.mark.parametrize("most", [0, 1, 2, 3])
@pytest.mark.parametrize("tau", [0.6, -1.0])
def test_acceptance_of_rows_with_few_tokens(mode, traversal, most, tau):
    """Drafts among them that copy their parent, and the step that the oracle takes."""
    rng = np.random.default_rng(most)
    B, N, L, k = 12, 9, 8, 3
    tau = float(np.float32(tau))
    committed = np.where(rng.random((B, L)) < 0.8, -1, 50).astype(np.int32)
    conf0, idx0 = table(rng, (B, L), k, most)
    conf, idx = table(rng, (B, N, L), k, most)
    parent = np.array([-1, -1, 0, 1, 1, 2, -1, 6, 3], np.int32)
    tokens = np.empty((B, N, L), np.int32)
    for b in range(B):
        for n in range(N):
            q = parent[n]
            s, C, I = (committed[b], conf0[b], idx0[b]) if q < 0 else (tokens[b, q], conf[b, q], idx[b, q])
            step = oracle.threshold_step(s, C, I, tau)
            tokens[b, n] = s if n in (0, 4) or step is None else step
            if n == 5:
                tokens[b, n] = np.where((s == -1) & (rng.random(L) < 0.5), I[:, 0], s)
    parents = np.broadcast_to(parent, (B, N)).copy()
    out = tsp.accept(cuda(conf), cuda(idx), cuda(tokens), cuda(parents), cuda(committed), cuda(conf0), cuda(idx0), tau, mode, traversal)
    check_accept(out, oracle.accept_batch(tokens, parents, committed, conf0, idx0, conf, idx, tau, mode, traversal))


def test_a_block_decoded_under_a_grammar():
    """Adjusted logits -> tree -> acceptance, step after step: positions that allow nothing stay masked, all others are
    filled, and what is accepted is what the oracles accept."""
    rng = np.random.default_rng(2)
    B, L, k, tau = 4, 12, 3, float(np.float32(0.6))
    conf, idx = adjusted_candidates(rng, B, L, k, 300)
    c, i = conf.cpu().numpy(), idx.cpu().numpy()
    state = np.full((B, L), -1, np.int32)
    for _ in range(L):
        tree = tsp.build_tree(cuda(state), conf, idx, tau, 2, 2, 2)
        n = tree["parent"].shape[1]
        drafts = [x.cpu().numpy() for x in (tree["tokens"], tree["parent"])]
        many = [x[:, None].expand(B, n, L, k).contiguous() for x in (conf, idx)]  # the model says the same of every draft
        out = tsp.accept(*many, tree["tokens"], tree["parent"], cuda(state), conf, idx, tau)
        ref = oracle.accept_batch(*drafts, state, c, i, *(x.cpu().numpy() for x in many), tau)
        check_accept(out, ref)
        left = (state == -1) & (i[..., 0] >= 0)
        assert ((ref["n_accepted"] > 0) == left.any(1)).all()
        state = ref["out_tokens"].astype(np.int32)
    assert ((state == -1) == (i[..., 0] < 0)).all()
