"""Rotary positions, head redistribution and windowed attention run together, as a layer of a sequence-parallel model runs them, and the windowed replay."""
from dataclasses import replace

import pytest
import torch

import window_util as wu
from paper_2605_07569_amd import hexi, workloads
from paper_2605_07569_amd.replay import ShardRun
from test_gpu_rope import freqs, turned

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


class Layer:
    """Two ranks hold parts of a sequence with all heads, fused [rows][nq + 2 nkv][d]; after the exchange each holds all rows of its own heads.  On one GPU
    the exchange is a copy between the ranks' buffers.  Everything is allocated here, so that a step can be captured."""

    def __init__(self, dtype, d, rows=(333, 367), nq=6, nkv=2, window=150, n_sink=5, start=1000, axes=2):
        self.dtype, self.d, self.rows, self.nq, self.nkv = dtype, d, rows, nq, nkv
        self.n, self.total = nq + 2 * nkv, sum(rows)
        self.segs = [[(start, rows[0])], [(start + rows[0], rows[1])]]
        self.range = [(start, self.total)]
        g = torch.Generator().manual_seed(11)
        self.x = [torch.randn(r, self.n, d, generator=g).to(dtype) for r in rows]
        self.d_o = torch.randn(self.total, nq, d, generator=g).to(dtype)
        self.freq, self.axis = freqs(d, axes)
        self.pos = torch.stack([torch.arange(self.total) // (7 * a + 1) for a in range(axes)]).to(torch.int32)
        self.window, self.n_sink, self.axes = window, n_sink, axes
        # rank r's heads: a third of the q heads on rank 0, the rest on rank 1, with the kv heads that they read
        cut = nq // 3
        per = nq // nkv
        self.q_heads = [list(range(cut)), list(range(cut, nq))]
        self.kv_heads = [sorted({h // per for h in hs}) for hs in self.q_heads]
        self.kv_of_q = [[ks.index(h // per) for h in hs] for hs, ks in zip(self.q_heads, self.kv_heads)]
        self.lists = [hs + [nq + k for k in ks] + [nq + nkv + k for k in ks] for hs, ks in zip(self.q_heads, self.kv_heads)]
        self.rotate = [1] * (nq + nkv) + [0] * nkv
        # gradients come back once for every rank that a kv head went to: each rank's into a buffer of its own
        self.device()

    def device(self):
        dev = dict(device=DEV)
        e = lambda *s, dtype=self.dtype: torch.full(s, float("nan"), dtype=dtype, **dev)
        self.rope = hexi.make_rope(self.d, self.freq, self.axis, n_axes=self.axes)
        self.win = hexi.make_window(self.window, self.n_sink)
        self.xd = [x.to(DEV) for x in self.x]
        ends = [0, self.rows[0], self.total]
        self.posd = [self.pos[:, a:b].contiguous().to(DEV) for a, b in zip(ends, ends[1:])]
        self.packed = [e(sum(len(h) for h in self.lists) * r * self.d) for r in self.rows]
        self.heads = [e(self.total, len(h), self.d) for h in self.lists]                 # what a rank has after the exchange
        self.g_heads = [e(self.total, len(h), self.d) for h in self.lists]
        self.back = [[e(r * len(h) * self.d) for h in self.lists] for r in self.rows]
        self.dx = [[torch.zeros(r, self.n, self.d, dtype=self.dtype, **dev) for _ in self.lists] for r in self.rows]
        self.out, self.state = [], []
        for r, (hs, ks) in enumerate(zip(self.q_heads, self.kv_heads)):
            a, b = len(hs), len(ks)
            h = self.heads[r]
            q, k, v = h[:, :a], h[:, a:a + b], h[:, a + b:]
            d_o = torch.zeros(self.total, len(self.lists[r]), self.d, dtype=self.dtype, **dev)[:, :a]      # (of q's strides)
            d_o.copy_(self.d_o[:, hs].to(DEV))
            desc = hexi.desc_for(q, k, self.d ** -0.5, self.kv_of_q[r])
            n = hexi.hexi_attn_win_workspace_bytes(desc, self.win, self.total, self.total)
            ws = torch.empty(n, dtype=torch.uint8, **dev) if n else None
            o, lse, delta = e(self.total, a, self.d), e(a, self.total, dtype=F32), e(a, self.total, dtype=F32)
            grads = [torch.zeros(self.total, m, self.d, dtype=self.dtype, **dev) for m in (a, b, b)]
            self.state.append((desc, q, k, v, d_o, o, lse, delta, grads, ws))
            self.out.append(o)

    def step(self):
        d = self.d
        for s, segs in enumerate(self.segs):
            hexi.hexi_rope_a2a_pack(self.rope, segs, self.xd[s], self.packed[s], self.lists, self.rotate, positions=self.posd[s])
        for r, lst in enumerate(self.lists):      # the exchange
            row = 0
            for s, rows in enumerate(self.rows):
                at = sum(len(h) for h in self.lists[:r]) * rows * d
                self.heads[r][row:row + rows].view(-1).copy_(self.packed[s][at:at + len(lst) * rows * d])
                row += rows
        for r, (desc, q, k, v, d_o, o, lse, delta, (dq, dk, dv), ws) in enumerate(self.state):
            hexi.hexi_attn_win_fwd_chunk(desc, self.win, self.range, self.range, q, k, v, o, lse, workspace=ws)
            if self.dtype == F32:
                dq.zero_()
            hexi.hexi_attn_win_bwd_chunk(desc, self.win, self.range, self.range, q, k, v, o, d_o, lse, delta, dq, dk, dv, flags=hexi.HEXI_COMPUTE_DELTA)
            torch.cat([dq, dk, dv], 1, out=self.g_heads[r])
            row = 0
            for s, rows in enumerate(self.rows):
                self.back[s][r].copy_(self.g_heads[r][row:row + rows].reshape(-1))
                row += rows
        for s, segs in enumerate(self.segs):
            for r, lst in enumerate(self.lists):
                hexi.hexi_rope_a2a_unpack(self.rope, segs, self.back[s][r], self.dx[s][r], [lst], self.rotate, positions=self.posd[s])

    def results(self):
        return [t.clone() for t in self.out + [sum(g.float() for g in per) for per in self.dx]]

    def wanted(self):
        """The same in float64, by autograd over the definition."""
        nq, nkv = self.nq, self.nkv
        x = torch.cat(self.x).double().requires_grad_()
        y, _ = turned(x, self.pos, self.freq, self.axis, False, False)
        q, k, v = y[:, :nq], y[:, nq:nq + nkv], x[:, nq + nkv:]
        p = torch.arange(self.total) + self.range[0][0]
        seen = (p[None] <= p[:, None]) & ((p[:, None] - p[None] < self.window) | (p[None] < self.n_sink))
        o = []
        for h in range(nq):
            s = (q[:, h] @ k[:, h // (nq // nkv)].T * self.d ** -0.5).masked_fill(~seen, float("-inf"))
            o.append(torch.softmax(s, 1) @ v[:, h // (nq // nkv)])
        o = torch.stack(o, 1)
        (o * self.d_o.double()).sum().backward()
        return [o[:, hs].detach() for hs in self.q_heads] + list(x.grad.split(self.rows))


# relative L2 allowed: rotated q and k are rounded once (2^-8 / sqrt(12) of each element's rms at worst, both of them in a score of about 1: 2e-3 of P), then as for the
# attention alone (under 5e-3), gradients through P and dP both and rounded twice more on the way: 7e-3 and 1.2e-2; fp32: 1e-5 and 2e-5
REL = {BF16: (7e-3, 1.2e-2), F32: (1e-5, 2e-5)}


@pytest.mark.parametrize("dtype,d,kw", [(BF16, 128, {}), (F32, 64, {}), (F32, 128, dict(rows=(1, 2), nq=3, nkv=1)),
                                        (BF16, 64, dict(rows=(64, 449), nq=12, nkv=4, window=10 ** 9, n_sink=0, axes=1)),
                                        (BF16, 128, dict(rows=(5, 300), window=1, n_sink=1003, nq=6, nkv=1))], ids=str)
def test_layer_forward_and_backward(dtype, d, kw):
    layer = Layer(dtype, d, **kw)
    layer.step()
    torch.cuda.synchronize()
    for i, (got, want) in enumerate(zip(layer.results(), layer.wanted())):
        rel = float((got.double().cpu() - want).norm() / want.norm())
        print(f"\n    result {i}: rel-L2 {rel:.2e}", flush=True)
        assert rel <= REL[dtype][i >= 2]


def test_layer_captured_and_replayed():
    layer = Layer(BF16, 128)
    layer.step()
    torch.cuda.synchronize()
    want = layer.results()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step()
    for _ in range(3):
        for t in layer.out + [g for per in layer.dx for g in per]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(layer.results(), want))
        other = Layer(BF16, 128)      # the program's own work between the replays
        other.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(other.results(), want))


@pytest.mark.parametrize("dtype,rel", [("bf16", 5e-3), ("f32", 1e-5)])
def test_windowed_replay_over_the_ring_and_over_one_chunk(dtype, rel):
    """A zigzag shard: the ring of all chunks and the one chunk of the keys that its rows see give what the definition gives."""
    total, ranks, window, n_sink = 1536, 4, 200, 9
    w = workloads.Workload("ring", dtype, 4, 2, 64, total, workloads.zigzag_segs(1, ranks, total), [workloads.zigzag_segs(r, ranks, total) for r in range(ranks)])
    inputs = workloads.make_inputs(w)
    one = workloads.windowed(w, window, n_sink)
    assert one.chunks == [[(0, 384), (953, 391)]]
    c = wu.Case("ring", w.q_segs, [(0, total)], window, n_sink, nq=4, nkv=2)
    x = dict(q=inputs["q"], k=inputs["k"], v=inputs["v"], d_o=inputs["d_o"])
    o, lse, bo, bl = wu.forward(c, x, F32)
    for run_of in (w, replace(w, chunks=w.chunks[::-1]), one):
        run = ShardRun(run_of, inputs, window=hexi.make_window(window, n_sink), fused_merge=run_of is not w)
        run.step()
        torch.cuda.synchronize()
        n = len(run_of.chunks)
        wu.within("o", run.o, o, n * bo, rel)
        wu.within("lse", run.lse, lse, n * bl)
        want = wu.backward(c, x, run.o.cpu(), run.lse.cpu(), F32)
        wu.within("dq", run.dq, *(z * f for z, f in zip(want["dq"], (1, n))), rel)
        for name, parts in (("dk", run.dk), ("dv", run.dv)):
            got = torch.zeros_like(want[name][0])
            for segs, part in zip(run_of.chunks, parts):
                row = 0
                for s, m in segs:
                    got[s:s + m] += part[row:row + m].double().cpu()
                    row += m
            wu.within(name, got, *want[name], rel)
