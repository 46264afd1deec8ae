"""A serving step in 8 bits as a server runs it: projection, append, attention, output projection and logits, several steps in
a row, captured and replayed, on other streams; and what the binding refuses."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_27514_amd as tsp
from helpers import cuda
from oracle import eight
from test_gpu_eight import BF, E4, E8, U8, bf, bytes_of, check_append, f64

pytestmark = pytest.mark.gpu


class Server:
    """A small model's layer and head, a paged cache of B sequences, a denoising block of T tokens per step."""

    B, T, Hq, Hkv, D, V, ps, sb, columns = 3, 8, 4, 2, 64, 1000, 32, 16, 15

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        hidden = self.Hq * self.D
        self.w_qkv = tsp.quantize8(bf(rng.standard_normal((hidden, (self.Hq + 2 * self.Hkv) * self.D)) / hidden ** 0.5))
        self.w_o = tsp.quantize8(bf(rng.standard_normal((hidden, hidden)) / hidden ** 0.5))
        self.w_head = tsp.quantize8(bf(3 * rng.standard_normal((hidden, self.V)) / hidden ** 0.5))
        pages = self.B * self.columns
        self.table = cuda(rng.permutation(pages).reshape(self.B, -1).astype(np.int32))
        self.cache = (*(torch.zeros(pages, self.ps, self.Hkv, self.D, dtype=E4, device="cuda") for _ in range(2)),
                      *(torch.full((pages, self.ps // self.sb, self.Hkv), 127, dtype=U8, device="cuda").view(E8) for _ in range(2)))
        k, v = (bf(rng.standard_normal((self.B, 300, self.Hkv, self.D))) for _ in range(2))
        tsp.paged_append8(k, v, *self.cache, self.table, torch.zeros(self.B, dtype=torch.int32, device="cuda"))
        self.x = bf(rng.standard_normal((self.B, self.T, hidden)))
        self.start = cuda(np.array([0, 5, 300], np.int32))
        self.n_new = cuda(np.array([8, 3, 7], np.int32))

    def step(self):
        B, T, Hq, Hkv, D = self.B, self.T, self.Hq, self.Hkv, self.D
        qkv = tsp.linear8(self.x, *self.w_qkv)
        q, k, v = (t.view(B, T, -1, D) for t in qkv.split([Hq * D, Hkv * D, Hkv * D], -1))
        q = tsp.paged_append8(k, v, *self.cache, self.table, self.start, q=q, n_new=self.n_new)
        a = tsp.paged_attn8(q, *self.cache, self.table, self.start + self.n_new, n_new=self.n_new)
        h = self.x.clone()
        tsp.linear8(a.view(B, T, Hq * D), *self.w_o, y=h, accumulate=True)
        logits = tsp.linear8(h, *self.w_head).view(B * T, self.V)
        conf, idx = tsp.confidence_topk(logits, 3)
        return dict(qkv=qkv, q=q, a=a, h=h, logits=logits, conf=conf, idx=idx)

    def advance(self, out):
        """The next step's inputs, from this one's."""
        self.start.add_(self.n_new)
        self.x.copy_((out["h"].float() * 0.7).to(BF))


def test_steps_against_the_oracle():
    """Each operator's result against the oracle on the same inputs, over steps that build on each other."""
    s = Server(1)
    tsp.device_status()
    qw = [(f64(w).transpose(0, 2, 1).reshape(-1, w.shape[1]), bytes_of(z).T) for w, z in (s.w_qkv, s.w_o, s.w_head)]
    near = lambda got, ref, size: (np.abs(f64(got) - ref) <= 2.0 ** -10 * size + 2.0 ** -8 * np.abs(ref)).all()  # noqa: E731
    for _ in range(4):
        before = [f64(t) if t.dtype == E4 else bytes_of(t) for t in s.cache]
        start, n_new, table, x = (t.clone() for t in (s.start, s.n_new, s.table, s.x))
        start, n_new, table, x = start.cpu().numpy(), n_new.cpu().numpy(), table.cpu().numpy(), f64(x).reshape(s.B * s.T, -1)
        out = s.step()
        assert tsp.device_status() == 0
        qkv = f64(out["qkv"])
        assert near(out["qkv"].view(s.B * s.T, -1), *eight.linear8(x, *qw[0]))
        q, k, v = (t.reshape(s.B, s.T, -1, s.D) for t in np.split(qkv, [s.Hq * s.D, (s.Hq + s.Hkv) * s.D], -1))
        ref, pools, exact = eight.paged_append8(q, k, v, before, table, start, n_new)
        size = np.abs(q) + np.abs(np.roll(q, s.D // 2, -1))
        check_append(s.cache, out["q"], (ref, size), pools, exact, qkv, 500000.0)
        now = [f64(t) if t.dtype == E4 else bytes_of(t) for t in s.cache]
        ra, weight = oracle.paged_attention(f64(out["q"]), eight.paged_values(now[0], now[2]), eight.paged_values(now[1], now[3]), table,
                                            start + n_new, n_new=n_new)
        assert (np.abs(f64(out["a"]) - ra) <= 2.0 ** -10 * weight + 2.0 ** -8 * np.abs(ra)).all()
        y, size = eight.linear8(f64(out["a"]).reshape(s.B * s.T, -1), *qw[1])
        assert near(out["h"].view(s.B * s.T, -1), y + x, size)
        assert near(out["logits"], *eight.linear8(f64(out["h"]).reshape(s.B * s.T, -1), *qw[2]))
        s.advance(out)


def test_a_captured_step_replays_bit_for_bit():
    """The whole step in a graph, replayed over steps that change its inputs in place, with eager work and
    synchronisation between, against a second server that runs eagerly."""
    s, e = Server(2), Server(2)
    s.step()  # warm
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = s.step()
    torch.cuda.synchronize()
    for a, b in zip(s.cache, e.cache):
        a.view(U8).copy_(b.view(U8))
    for n in range(4):
        for t in out.values():
            t.fill_(1)
        graph.replay()
        want = e.step()
        torch.cuda.synchronize()
        for name in out:
            assert torch.equal(out[name], want[name]), (n, name)
        for a, b in zip(s.cache, e.cache):
            assert torch.equal(a.view(U8), b.view(U8)), n
        s.advance(out)
        e.advance(want)
        torch.cuda.synchronize()


def test_two_graphs_with_their_own_workspaces():
    """Calls whose keys and whose k are split, captured twice over different inputs and replayed in turn."""
    rng = np.random.default_rng(3)
    graphs = []
    for n, M in ((3000, 3), (4500, 100)):
        q = bf(rng.standard_normal((2, 1, 4, 128)))
        cache = (*(torch.from_numpy(rng.standard_normal((300, 32, 2, 128))).to(E4).cuda() for _ in range(2)),
                 *(torch.full((300, 2, 2), 126, dtype=U8, device="cuda").view(E8) for _ in range(2)))
        table = cuda(rng.permutation(300).reshape(2, -1).astype(np.int32))
        lens = cuda(np.array([n, 700], np.int32))
        x, w = bf(rng.standard_normal((M, 4096))), tsp.quantize8(bf(rng.standard_normal((4096, 256))))
        ws = torch.empty(max(1, tsp.paged_attn8_workspace_size(q, *cache, table)), dtype=U8, device="cuda")
        lws = torch.empty(tsp.linear8_workspace_size(M, 4096, 256), dtype=U8, device="cuda")
        call = lambda q=q, cache=cache, table=table, lens=lens, x=x, w=w, ws=ws, lws=lws: (  # noqa: E731
            tsp.paged_attn8(q, *cache, table, lens, workspace=ws), tsp.linear8(x, *w, workspace=lws))
        want = [t.clone() for t in call()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out, want))
    for _ in range(3):
        for graph, out, _ in graphs:
            for t in out:
                t.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, out, want in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_other_streams():
    s, e = Server(4), Server(4)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    want = e.step()
    with torch.cuda.stream(stream):
        got = s.step()
    stream.synchronize()
    for name in got:
        assert torch.equal(got[name], want[name]), name
    x, w = bf(np.ones((40, 256))), bf(np.random.default_rng(5).standard_normal((256, 136)))
    torch.cuda.synchronize()
    w8, scale = tsp.quantize8(w, stream=stream)
    y = tsp.linear8(x, w8, scale, stream=stream)
    stream.synchronize()
    assert torch.equal(y, tsp.linear8(x, *tsp.quantize8(w)))


def test_the_binding_refuses():
    s = Server(6)
    q, k = (torch.zeros(3, 8, h, 64, dtype=BF, device="cuda") for h in (4, 2))
    n = torch.zeros(3, dtype=torch.int32, device="cuda")
    kp, vp, ks, vs = s.cache
    for bad in ((kp.view(U8), vp, ks, vs), (kp, vp[:, :16], ks, vs), (kp, vp, ks.view(U8), vs), (kp, vp, ks[:, :, :1], vs), (kp, vp, ks, vs[:5]),
                (kp.float(), vp, ks, vs), (kp, vp, torch.zeros(45, 3, 2, dtype=U8, device="cuda").view(E8), vs), (kp.cpu(), vp, ks, vs)):
        with pytest.raises((TypeError, ValueError)):
            tsp.paged_append8(k, k, *bad, s.table, n)
        with pytest.raises((TypeError, ValueError)):
            tsp.paged_attn8(q, *bad, s.table, n)
    with pytest.raises(tsp.TrajSpecError):  # a scale of 128 tokens
        wide = torch.zeros(2, 128, 2, 64, dtype=E4, device="cuda")
        one = torch.zeros(2, 1, 2, dtype=U8, device="cuda").view(E8)
        tsp.paged_attn8(q, wide, wide, one, one, s.table, n)
    w8, scale = s.w_o
    x = torch.zeros(2, 256, dtype=BF, device="cuda")
    for bad in ((x.float(), w8, scale), (x[:, :120], w8, scale), (x, w8.view(U8), scale), (x, w8[:2], scale), (x, w8, scale[:1]),
                (x, w8.transpose(1, 2), scale), (x.cpu(), w8, scale), (x.t(), w8, scale)):
        with pytest.raises((TypeError, ValueError)):
            tsp.linear8(*bad)
    with pytest.raises(ValueError):
        tsp.linear8(x, w8, scale, accumulate=True)
    with pytest.raises(ValueError):
        tsp.linear8(x, w8, scale, y=torch.zeros(3, 256, dtype=BF, device="cuda"))
    with pytest.raises((TypeError, ValueError)):
        tsp.quantize8(torch.zeros(256, 128, device="cuda"))
    with pytest.raises((TypeError, ValueError)):
        tsp.quantize8(torch.zeros(256, 128, dtype=BF, device="cuda").t())
    with pytest.raises(tsp.TrajSpecError):
        tsp.quantize8(torch.zeros(100, 128, dtype=BF, device="cuda"))
