"""One GPU's share of an MoE layer in 8 bits, from the residual stream to the layer's output: norm with the residual's addition,
gate with groups, send buffer of packed 8-bit rows, expert FFN on them, weighted combine.

    python examples/fp8_share.py [--tokens 4096] [--hidden 2048] [--inner 1408] [--experts 64] [--top 6] [--groups 8] [--top-groups 4]

On one GPU the two all-to-alls are the identity: what it sends is what it receives.  With more, the rows of `send` travel as
they are (values and scales together, about half the bytes of bf16), and `out` travels back.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2410_17043_amd as P  # noqa: E402

BLOCK = 128


def quantize_weight(w):
    """[n, K] -> e4m3 [n, K] and its scale bytes [n / 128, K / 128]: once, when the model is loaded."""
    n, K = w.shape
    blocks = w.float().reshape(n // BLOCK, BLOCK, K // BLOCK, BLOCK)
    mantissa, exponent = torch.frexp(blocks.abs().amax((1, 3)) / 448.0)       # smallest power of two that is no less
    b = (exponent - (mantissa == 0.5).to(exponent.dtype) + 127).clamp(1, 254)
    q = (blocks / torch.ldexp(torch.ones_like(mantissa), b - 127)[:, None, :, None]).reshape(n, K).to(torch.float8_e4m3fn)
    return q.contiguous(), b.to(torch.uint8).contiguous()


class Fp8Share:
    """Buffers, contexts and bound calls of a layer of T tokens, made once; `x` and `residual` are the inputs, `y` and `residual_out` the results."""

    def __init__(self, T, H, F, E, k, act, experts, w_gate, gamma, rule, select_bias=None, renorm=1, eps=1e-6):
        dev = w_gate.device
        bf16 = dict(dtype=torch.bfloat16, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        S, pitch = T * k, P.moe_fp8_row_bytes(H)
        e2g, order = [0] * E, [0]                                              # all experts here
        self.x, self.residual = torch.zeros(T, H, **bf16), torch.zeros(T, H, **bf16)
        self.residual_out, self.normed, self.y = torch.empty(T, H, **bf16), torch.empty(T, H, **bf16), torch.empty(T, H, **bf16)
        self.rows = torch.empty(T, pitch, dtype=torch.uint8, device=dev)
        self.idx, self.w = torch.empty(T, k, **i32), torch.empty(T, k, dtype=torch.float32, device=dev)
        self.send = torch.empty(S, pitch, dtype=torch.uint8, device=dev)
        self.slot_to_row, self.row_to_slot = torch.empty(S, **i32), torch.empty(S, **i32)
        self.seg_offset, self.seg_expert = torch.empty(E + 1, **i32), torch.empty(E, **i32)
        self.out = torch.empty(S, H, **bf16)
        gate = P.MoeCtx(T, H, E, k, 1, "bf16", renorm)
        wire = P.MoeCtx(T, pitch // 2, E, k, 1, "bf16", renorm)                # packed rows are rows of pitch / 2 16-bit words
        gate_ws = torch.empty(P.moe_route_grouped_workspace_bytes(gate), dtype=torch.uint8, device=dev)
        ffn_ws = torch.empty(P.moe_ffn_fp8_workspace_bytes(S, H, F, act), dtype=torch.uint8, device=dev)
        self.calls = [
            P.bind_norm_fp8(self.x, self.residual, gamma, eps, self.residual_out, self.normed, self.rows),
            P.bind_route_grouped(gate, self.normed, w_gate, rule, select_bias, self.idx, self.w, gate_ws),
            P.bind_dispatch(wire, self.rows.view(torch.bfloat16), self.idx, e2g, order, self.send.view(torch.bfloat16), self.slot_to_row, self.row_to_slot,
                            self.seg_offset, self.seg_expert),
            P.bind_expert_ffn_fp8(self.send, S, self.seg_offset, self.seg_expert, E, experts, H, F, act, self.out, ffn_ws),
            P.bind_combine(gate, self.out, self.slot_to_row, self.w, None, self.y)]
        self.names = ["norm", "gate", "dispatch", "ffn", "combine"]

    def run(self, stream=None):
        """On the stream that was current when the share was made, or on this one (a handle) from now on; may be captured into a graph."""
        for call in self.calls:
            call(stream)
        return self.y


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("tokens", 4096), ("hidden", 2048), ("inner", 1408), ("experts", 64), ("top", 6), ("groups", 8), ("top-groups", 4), ("steps", 20)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    g = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    experts = []
    for _ in range(a.experts):
        e = {}
        for name, n, K in (("1", a.inner, a.hidden), ("_up", a.inner, a.hidden), ("_down", a.hidden, a.inner)):
            e["w" + name], e["s" + name] = quantize_weight(randn(n, K) * 0.02)
        experts.append(e)
    rule = P.gate_rule(P.SCORE_SIGMOID, a.groups, a.top_groups, P.GROUP_TOP2)
    share = Fp8Share(a.tokens, a.hidden, a.inner, a.experts, a.top, P.ACT_SWIGLU, experts, (randn(a.experts, a.hidden) * 0.02).bfloat16(),
                     torch.ones(a.hidden, device="cuda", dtype=torch.bfloat16), rule, torch.zeros(a.experts, device="cuda"))
    share.x.copy_(randn(a.tokens, a.hidden))
    share.residual.copy_(randn(a.tokens, a.hidden))
    share.run()
    marks = [torch.cuda.Event(enable_timing=True) for _ in range(len(share.calls) + 1)]
    total = dict.fromkeys(share.names, 0.0)
    for _ in range(a.steps):
        marks[0].record()
        for call, mark in zip(share.calls, marks[1:]):
            call()
            mark.record()
        torch.cuda.synchronize()
        for i, name in enumerate(share.names):
            total[name] += marks[i].elapsed_time(marks[i + 1]) * 1e3 / a.steps
    print("  ".join("%s %.1f us" % (n, t) for n, t in total.items()), " together %.1f us" % sum(total.values()))
    print("y: %s, finite: %s" % (tuple(share.y.shape), bool(torch.isfinite(share.y).all())))


if __name__ == "__main__":
    main()
