"""The windowed backward on a stream given by its handle: the same workspace, and so the same sums in the same order, as on torch's current stream."""
import ctypes

import pytest
import torch

import window_util as wu
from paper_2605_07569_amd import hexi
from test_gpu_window import BF16, DEV, F32, REL, setup

pytestmark = pytest.mark.gpu


class Step:
    """A backward step that is cut into parts; what(...) runs it into buffers of its own."""

    def __init__(self, c, dtype, d=64):
        self.c, self.dtype, self.d = c, dtype, d
        self.x, self.dev, self.desc, self.window = setup(c, dtype, d, 31)
        ro, rl, _, _ = wu.forward(c, self.x, F32)
        self.o, self.lse = ro.float().to(DEV), rl.float().to(DEV)
        self.ref = wu.backward(c, self.x, ro.float(), rl.float(), dtype)
        self.need = hexi.hexi_attn_win_bwd_workspace_bytes(self.desc, self.window, c.lq, c.lc)
        assert self.need > 0

    def buffers(self):
        e = lambda *s, t=self.dtype: torch.zeros(s, dtype=t, device=DEV)
        c, d = self.c, self.d
        return dict(delta=e(c.nq, c.lq, t=F32), dq=e(c.lq, c.nq, d), dk=e(c.lc, c.nkv, d), dv=e(c.lc, c.nkv, d))

    def run(self, b, **kw):
        c = self.c
        hexi.hexi_attn_win_bwd_chunk(self.desc, self.window, c.q_segs, c.kv_segs, self.dev["q"], self.dev["k"], self.dev["v"], self.o, self.dev["d_o"], self.lse, b["delta"], b["dq"],
                                     b["dk"], b["dv"], flags=hexi.HEXI_COMPUTE_DELTA, **kw)
        return b

    def check(self, b):
        for name in ("dq", "dk", "dv"):
            wu.within(name, b[name], *self.ref[name], max(REL[self.dtype], 0 if self.dtype == F32 else REL[BF16]))


def same(a, b):
    return all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("c", [wu.PARTS[0], wu.PARTS[3]], ids=lambda c: c.name)
def test_the_same_bits_on_a_stream_given_by_hand(c, dtype):
    step = Step(c, dtype)
    want = step.run(step.buffers())
    torch.cuda.synchronize()
    step.check(want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    bufs = [step.buffers() for _ in range(3)]
    torch.cuda.synchronize()
    step.run(bufs[2], stream=torch.cuda.current_stream().cuda_stream)
    for again in range(3):      # on both at once
        for b in bufs[:2]:
            b["dq"].zero_()
        torch.cuda.synchronize()
        for b, s in zip(bufs, streams):
            step.run(b, stream=s.cuda_stream)
        torch.cuda.synchronize()
        assert all(same(b, want) for b in bufs), again


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_stream_given_by_hand_inside_a_graph(dtype):
    """A branch of a captured graph, its stream given by its handle, among eager calls on the same stream."""
    step = Step(wu.PARTS[0], dtype)
    want = step.run(step.buffers())
    captured, eager, side = step.buffers(), step.buffers(), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        captured["dq"].zero_()
        side.wait_stream(main)
        step.run(captured, stream=side.cuda_stream)
        main.wait_stream(side)
    for _ in range(4):
        for name in ("dk", "dv"):
            captured[name].fill_(float("nan"))
        eager["dq"].zero_()
        torch.cuda.synchronize()
        graph.replay()
        step.run(eager, stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert same(captured, want) and same(eager, want)


def test_a_capture_that_torch_does_not_know_of_takes_no_memory():
    """torch would hand the memory out again while the graph lives: the call does without."""
    step = Step(wu.PARTS[0], F32)
    hip, stream, graph, program = hexi.load(), torch.cuda.Stream(), ctypes.c_void_p(), ctypes.c_void_p()
    handle = ctypes.c_void_p(stream.cuda_stream)
    b = step.buffers()
    torch.cuda.synchronize()
    count = lambda: torch.cuda.memory_stats()["allocation.all.allocated"]
    assert hip.hipStreamBeginCapture(handle, 1) == 0
    before = count()
    step.run(b, stream=stream.cuda_stream)
    taken = count() - before
    assert hip.hipStreamEndCapture(handle, ctypes.byref(graph)) == 0
    assert taken == 0
    assert hip.hipGraphInstantiate(ctypes.byref(program), graph, None, None, ctypes.c_size_t(0)) == 0
    for _ in range(3):
        for name in ("dk", "dv"):
            b[name].fill_(float("nan"))
        b["dq"].zero_()
        torch.cuda.synchronize()
        assert hip.hipGraphLaunch(program, handle) == 0
        torch.cuda.synchronize()
        step.check(b)
    assert hip.hipGraphExecDestroy(program) == 0 and hip.hipGraphDestroy(graph) == 0
