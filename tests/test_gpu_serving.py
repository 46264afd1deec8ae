"""The paged cache and the adjusted candidates as a server uses them: several decoding steps in a row, captured and
replayed, on other streams; and what the binding refuses."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import CONF_ATOL, cuda

pytestmark = pytest.mark.gpu
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HALF_STEP = 2.0 ** -8


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def bf(x):
    return cuda(np.asarray(x, dtype=np.float32), BF)


class Server:
    """A small model's layer and head, a paged cache of B sequences, a denoising block of T tokens per step."""

    B, T, Hq, Hkv, D, V, ps, columns = 3, 8, 4, 2, 64, 1000, 16, 30

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        hidden = self.Hq * self.D
        self.w_qkv = bf(rng.standard_normal((hidden, (self.Hq + 2 * self.Hkv) * self.D)) / hidden ** 0.5)
        self.w_head = bf(3 * rng.standard_normal((hidden, self.V)) / hidden ** 0.5)
        pages = self.B * self.columns
        self.table = cuda(rng.permutation(pages).reshape(self.B, -1).astype(np.int32))
        self.kp, self.vp = (bf(rng.standard_normal((pages, self.ps, self.Hkv, self.D))) for _ in range(2))
        self.x = bf(rng.standard_normal((self.B, self.T, hidden)))
        self.start = cuda(np.array([0, 5, 300], np.int32))
        self.n_new = cuda(np.array([8, 3, 7], np.int32))
        self.history = cuda(rng.integers(-1, self.V, (self.B, 20)).astype(np.int32))
        self.penalty = [cuda(rng.uniform(lo, hi, self.B).astype(np.float32)) for lo, hi in ((1, 2), (0, 0.5), (0, 0.5))]
        self.bias_ids = cuda(rng.integers(0, self.V, (self.B, 3)).astype(np.int32))
        self.bias = cuda(rng.standard_normal((self.B, 3)).astype(np.float32))
        self.mask = cuda(rng.integers(-2 ** 31, 2 ** 31, (4, -(-self.V // 32))).astype(np.int32))
        self.mask_index = cuda(rng.integers(-1, 4, self.B * self.T).astype(np.int32))
        self.tokens = cuda(rng.integers(-1, self.V, (self.B, 2, self.T)).astype(np.int32))

    def step(self):
        """Projection, append, attention, head, candidates: every intermediate."""
        B, T, Hq, Hkv, D = self.B, self.T, self.Hq, self.Hkv, self.D
        qkv = tsp.linear(self.x, self.w_qkv)
        q, k, v = (t.view(B, T, -1, D) for t in qkv.split([Hq * D, Hkv * D, Hkv * D], -1))
        lens = self.start + self.n_new
        q = tsp.paged_append(k, v, self.kp, self.vp, self.table, self.start, q=q, n_new=self.n_new)
        a = tsp.paged_attn(q, self.kp, self.vp, self.table, lens)
        logits = tsp.linear(a.view(B, T, Hq * D), self.w_head).view(B * T, self.V)
        r, f, p = self.penalty
        conf, idx = tsp.confidence_topk_adjusted(logits, 3, T, history=self.history, repetition=r, frequency=f, presence=p,
                                                 bias_ids=self.bias_ids, bias=self.bias, mask=self.mask, mask_index=self.mask_index)
        # a draft of one step from the block's own candidates, and the next tree
        acc = tsp.accept(conf.repeat_interleave(2, 0), idx.repeat_interleave(2, 0), self.tokens,
                         torch.full((B, 2), -1, dtype=I32, device="cuda"), self.tokens[:, 0].contiguous(), conf.view(B, T, 3),
                         idx.view(B, T, 3), 0.3)
        tree = tsp.build_tree(acc["out_tokens"], conf.view(B, T, 3), idx.view(B, T, 3), 0.3, 2, 2, 2)
        return dict(qkv=qkv, q=q, a=a, logits=logits, conf=conf, idx=idx, kp=self.kp, vp=self.vp, tokens=tree["tokens"], leaf=acc["leaf"])

    def advance(self, out):
        """The next step's inputs, from this one's."""
        self.start.add_(self.n_new)
        self.history.copy_(torch.cat([self.history, out["idx"].view(self.B, -1)[:, :5]], 1)[:, 5:])
        self.x.copy_((out["a"].view_as(self.x).float() + 0.5 * self.x.float()).to(BF))


def test_decoding_steps_against_the_oracle():
    """Each operator's result against the oracle on the same inputs, over steps that build on each other."""
    s = Server(1)
    tsp.device_status()
    for _ in range(3):
        before = f64(s.kp), f64(s.vp)
        start, n_new, table, history = (t.cpu().numpy().copy() for t in (s.start, s.n_new, s.table, s.history))
        out = s.step()
        assert tsp.device_status() == 0
        qkv = f64(out["qkv"])
        q, k, v = (x.reshape(s.B, s.T, -1, s.D) for x in np.split(qkv, [s.Hq * s.D, (s.Hq + s.Hkv) * s.D], -1))
        rq, rk, rv = oracle.paged_append(q, k, v, *before, table, start, n_new)
        for got, ref in ((out["q"], rq), (s.kp, rk)):
            e = 2.0 ** -20 * 2 * np.abs(qkv).max()
            assert (np.abs(f64(got) - ref) <= HALF_STEP * (np.abs(ref) + e) + e).all()
        assert np.array_equal(f64(s.vp), rv)
        ra, weight = oracle.paged_attention(f64(out["q"]), f64(s.kp), f64(s.vp), table, start + n_new)
        assert (np.abs(f64(out["a"]) - ra) <= (HALF_STEP + 2.0 ** -10) * weight + HALF_STEP * np.abs(ra)).all()
        r, f, p = (t.cpu().numpy() for t in s.penalty)
        rc, ri = oracle.confidence_topk_adjusted(out["logits"].float().cpu().numpy(), 3, s.T, history=history, repetition=r, frequency=f,
                                                 presence=p, bias_ids=s.bias_ids.cpu().numpy(), bias=s.bias.cpu().numpy(),
                                                 mask=s.mask.cpu().numpy().view(np.uint32), mask_index=s.mask_index.cpu().numpy())
        assert np.array_equal(out["idx"].cpu().numpy(), ri)
        assert np.abs(out["conf"].cpu().numpy() - rc).max() <= CONF_ATOL
        s.advance(out)


def test_a_captured_step_replays_bit_for_bit():
    """The whole step in a graph, replayed over steps that change its inputs in place, with eager work and
    synchronisation between, against a second server that runs eagerly."""
    s, e = Server(2), Server(2)
    s.step()  # warm
    s.kp.copy_(e.kp)
    s.vp.copy_(e.vp)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = s.step()
    torch.cuda.synchronize()
    s.kp.copy_(e.kp)
    s.vp.copy_(e.vp)
    for n in range(4):
        for t in out.values():
            if t is not s.kp and t is not s.vp:
                t.fill_(1)
        graph.replay()
        want = e.step()
        torch.cuda.synchronize()
        for name in out:
            assert torch.equal(out[name], want[name]), (n, name)
        s.advance(out)
        e.advance(want)
        torch.cuda.synchronize()


def test_two_graphs_of_split_calls_with_their_own_workspaces():
    """Calls whose keys are split and whose rows are split, captured twice over different inputs and replayed in turn."""
    rng = np.random.default_rng(3)
    graphs = []
    for n in (3000, 4500):
        q = bf(rng.standard_normal((2, 1, 4, 128)))
        kp, vp = (bf(rng.standard_normal((300, 32, 2, 128))) for _ in range(2))
        table = cuda(rng.permutation(300).reshape(2, -1).astype(np.int32))
        lens = cuda(np.array([n, 700], np.int32))
        logits = bf(rng.standard_normal((2, 50000)))
        hist = cuda(rng.integers(0, 50000, (2, 3000)).astype(np.int32))
        r = cuda(np.array([1.5, 1.1], np.float32))

        def run():
            return (tsp.paged_attn(q, kp, vp, table, lens),) + tsp.confidence_topk_adjusted(logits, 4, 1, history=hist, repetition=r)

        want = [t.clone() for t in run()]
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            out = run()
        graphs.append((g, out, want, (q, kp, vp, table, lens, logits, hist, r)))
    for rep in range(3):
        for g, out, want, _ in graphs:
            for t in out:
                t.fill_(0)
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b), rep


def test_calls_on_other_streams():
    """Outputs and workspaces of a call on a stream are that stream's: runs side by side give what each gives alone."""
    servers = [Server(4), Server(5)]
    want = [{n: t.clone() for n, t in s.step().items()} for s in servers]
    streams = [torch.cuda.Stream() for _ in servers]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, stream in zip(servers, streams):
            lens = s.start + s.n_new
            stream.wait_stream(torch.cuda.current_stream())
            a = tsp.paged_attn(want[servers.index(s)]["q"], s.kp, s.vp, s.table, lens, stream=stream)
            r, f, p = s.penalty
            c = tsp.confidence_topk_adjusted(want[servers.index(s)]["logits"], 3, s.T, history=s.history, repetition=r, frequency=f, presence=p,
                                             bias_ids=s.bias_ids, bias=s.bias, mask=s.mask, mask_index=s.mask_index, stream=stream)
            got.append((a, *c, lens))
        torch.cuda.synchronize()
        for (a, conf, idx, _), w in zip(got, want):
            assert torch.equal(a, w["a"]) and torch.equal(conf, w["conf"]) and torch.equal(idx, w["idx"])


def test_what_the_binding_refuses():
    kp = torch.zeros(4, 16, 2, 64, dtype=BF, device="cuda")
    q = torch.zeros(2, 1, 4, 64, dtype=BF, device="cuda")
    k = torch.zeros(2, 1, 2, 64, dtype=BF, device="cuda")
    table = torch.zeros(2, 2, dtype=I32, device="cuda")
    n = torch.zeros(2, dtype=I32, device="cuda")

    def attn(**kw):
        a = dict(q=q, k_pages=kp, v_pages=kp, page_table=table, lens=n)
        return tsp.paged_attn(**{**a, **kw})

    def append(**kw):
        a = dict(k=k, v=k, k_pages=kp, v_pages=kp.clone(), page_table=table, start=n)
        return tsp.paged_append(**{**a, **kw})

    for call in (attn, append):
        for bad in (dict(k_pages=kp.float()), dict(v_pages=kp.cpu()), dict(page_table=table.long()), dict(page_table=table.cpu())):
            with pytest.raises(TypeError):
                call(**bad)
        for bad in (dict(k_pages=kp[:3]), dict(k_pages=kp.transpose(1, 2)), dict(k_pages=kp[..., ::2], v_pages=kp[..., ::2]),
                    dict(page_table=table[:1]), dict(page_table=table[0]),
                    dict(k_pages=kp[..., :32], v_pages=kp[..., :32])):
            with pytest.raises((ValueError, tsp.TrajSpecError)):
                call(**bad)
    with pytest.raises(TypeError):
        attn(q=q.float())
    with pytest.raises(TypeError):
        attn(lens=n.long())
    for bad in (dict(lens=n[:1]), dict(q=q[:, :, :, :32]), dict(out=q[:1]), dict(q=q.expand(2, 3, 4, 64))):
        with pytest.raises(ValueError):
            attn(**bad)
    room = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    for bad, err in ((room.cpu(), TypeError), (room[:1].expand(1 << 20), ValueError), (room[::2], ValueError)):
        with pytest.raises(err):
            attn(workspace=bad)
        with pytest.raises(err):
            tsp.confidence_topk_adjusted(torch.zeros(4, 100, dtype=BF, device="cuda"), 2, 2, history=table, workspace=bad)
    with pytest.raises(tsp.TrajSpecError, match="SHAPE"):
        attn(q=q[:, :, :3].contiguous())  # 3 query heads over 2
    for bad in (dict(start=n[:1]), dict(n_new=n[:1]), dict(q_out=q), dict(q=q, q_out=q[:1]), dict(v=k[:1]),
                dict(k=k.expand(2, 3, 2, 64), v=k.expand(2, 3, 2, 64))):
        with pytest.raises((ValueError, tsp.TrajSpecError)):
            append(**bad)
    logits = torch.zeros(4, 100, dtype=BF, device="cuda")
    hist = torch.zeros(2, 3, dtype=I32, device="cuda")
    pen = torch.ones(2, device="cuda")
    mask = torch.zeros(4, 4, dtype=I32, device="cuda")

    def adjusted(logits=logits, k=2, per=2, **kw):
        return tsp.confidence_topk_adjusted(logits, k, per, **kw)

    for bad in (dict(logits=logits.half()), dict(history=hist.long()), dict(history=hist, repetition=pen.double()), dict(mask=mask.long()),
                dict(history=hist.cpu()), dict(logits=logits.cpu())):
        with pytest.raises(TypeError):
            adjusted(**bad)
    for bad in (dict(per=0), dict(repetition=pen), dict(history=hist[:1]), dict(history=hist, presence=pen[:1]), dict(bias=pen[:, None]),
                dict(bias=pen[:, None], bias_ids=hist), dict(mask=mask[:3]), dict(mask=mask[:, :3]), dict(mask_index=hist[0]),
                dict(mask=mask, mask_index=hist[0]), dict(logits=logits.t()), dict(conf=torch.zeros(4, 3, device="cuda"))):
        with pytest.raises(ValueError):
            adjusted(**bad)
    for bad in (dict(k=0), dict(k=9)):
        with pytest.raises(tsp.TrajSpecError, match="ARG"):
            adjusted(**bad)


def test_more_sequences_than_are_split():
    """Batches beyond the largest that is split, lengths of none to some hundred."""
    rng = np.random.default_rng(6)
    B, H, D, ps = 2500, 1, 64, 16
    lens = rng.integers(0, 400, B).astype(np.int32)
    columns = 25
    pages = B * columns
    kp, vp = (torch.randn(pages, ps, H, D, device="cuda").to(BF) for _ in range(2))
    q = torch.randn(B, 1, H, D, device="cuda").to(BF)
    table = torch.randperm(pages, device="cuda").to(I32).view(B, columns)
    assert tsp.paged_attn_workspace_size(q, kp, vp, table) == 0
    out = tsp.paged_attn(q, kp, vp, table, cuda(lens))
    pick = rng.permutation(B)[:60]
    pick[0] = lens.argmin()
    ref, weight = oracle.paged_attention(f64(q)[pick], f64(kp), f64(vp), table.cpu().numpy()[pick], lens[pick])
    assert (np.abs(f64(out)[pick] - ref) <= (HALF_STEP + 2.0 ** -10) * weight + HALF_STEP * np.abs(ref) + 1e-30).all()
