"""A context's creation and its first calls, on the GPU."""
import pytest
import torch

from tests import harness as H
from tests.test_gpu_layer_few import Layer

pytestmark = pytest.mark.gpu
P = H.P
DEV = H.DEV


def test_creation_waits_for_no_stream():
    # what a serving loop does beside a step that is under way: a context for another batch size
    a = torch.randn(8192, 8192, device=DEV).bfloat16()
    b = torch.empty_like(a)
    torch.mm(a, a, out=b)
    torch.cuda.synchronize()
    for stream in (torch.cuda.default_stream(), torch.cuda.Stream()):
        done = torch.cuda.Event()
        with torch.cuda.stream(stream):
            for _ in range(400):                                             # a quarter of a second
                torch.mm(a, a, out=b)
            done.record()
            ctx = P.MoeCtx(64, 256, 8, 2, 1, "bf16")
            pending = not done.query()
        torch.cuda.synchronize()
        ctx.close()
        assert pending


def test_first_calls_in_memory_that_another_context_has_used():
    # ranks of another context's slots lie where this one's counters are, if its memory is the same
    for T in (1, 8, 40):
        c = Layer(T, 512, 384, 8, 2, renorm=1)
        c.ctx.close()
        other = P.MoeCtx(T + 40, 512, 8, 2, 1, "bf16")
        idx = torch.zeros(T + 40, 2, dtype=torch.int32, device=DEV)
        counts = [torch.empty(n, dtype=torch.int32, device=DEV) for n in (8, 1, 1)]
        P.moe_traffic(other, idx, [0] * 8, *counts)
        torch.cuda.synchronize()
        other.close()
        c.ctx = P.MoeCtx(T, 512, 8, 2, 1, "bf16", 1)
        c.check()


def test_first_call_in_a_graph():
    c = Layer(9, 512, 384, 8, 2, F_shared=128).device()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call = c.bind()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call(torch.cuda.current_stream().cuda_stream)
        for replay in (True, True, False, True, False, False, True):
            c.y.fill_(float("nan"))
            c.idx.fill_(-7)
            if replay:
                g.replay()
            else:
                call(side.cuda_stream)
            side.synchronize()
            c.check(gate=False)
            y, idx = c.y.clone(), c.idx.clone()
            c.bind()(side.cuda_stream)                                       # as an eager call has it
            side.synchronize()
            assert torch.equal(c.y, y) and torch.equal(c.idx, idx)
