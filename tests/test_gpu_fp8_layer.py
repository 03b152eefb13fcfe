"""The 8-bit share as a whole (examples/fp8_share.py) against the oracle: norm, gate, send buffer of packed rows, FFN, combine.

Tokens whose choice of experts hangs on rounding are left out (the gaps that decide are compared with the error of a logit, as in the
gate's own tests).  The tolerance is the FFN's (bf16): rows that round to 8 bits the other way because v is off by 2e-6 are one element in
10^5, and the combine rounds once more to bf16."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import fp8_layer as O
from tests import harness as H
from tests.test_gpu_fp8 import as_dtype, experts_to_dev, make_experts

pytestmark = pytest.mark.gpu
P = H.P
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("fp8_share", os.path.join(ROOT, "examples", "fp8_share.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("T,Hn,F,E,k,groups,top_groups,act,off", [
    (1, 256, 256, 8, 2, 4, 2, O.ACT_SWIGLU, 0), (50, 512, 384, 16, 4, 4, 2, O.ACT_SWIGLU, 0), (333, 256, 640, 24, 3, 6, 4, O.ACT_GELU_MLP, 2),
    (40, 384, 256, 12, 4, 3, 3, O.ACT_SILU_MLP, 10)])                          # ten of twelve out of service: dropped slots
def test_share_against_the_oracle(T, Hn, F, E, k, groups, top_groups, act, off):
    r = np.random.default_rng(T + E)
    experts = make_experts(r, E, Hn, F, act)
    w_gate, gamma = as_dtype(r.normal(size=(E, Hn)) * 0.05, "bf16"), as_dtype(1 + 0.1 * r.normal(size=Hn), "bf16")
    bias = (r.normal(size=E) * 0.1).astype(np.float32)
    bias[r.permutation(E)[:off]] = -np.inf
    share = example().Fp8Share(T, Hn, F, E, k, act, experts_to_dev(experts), H.dev(w_gate, "bf16"), H.dev(gamma, "bf16"),
                               P.gate_rule(P.SCORE_SIGMOID, groups, top_groups, P.GROUP_TOP2, 2.5), torch.from_numpy(bias).to(H.DEV))
    x, res = as_dtype(r.normal(size=(T, Hn)), "bf16"), as_dtype(r.normal(size=(T, Hn)) * 2, "bf16")
    share.x.copy_(H.dev(x, "bf16"))
    share.residual.copy_(H.dev(res, "bf16"))
    y = H.host(share.run()).astype(np.float64)
    s = as_dtype((x + res).astype(np.float32), "bf16")
    assert np.array_equal(H.host(share.residual_out).astype(np.float64), s)
    v = O.norm(s, gamma, 1e-6)
    logits = H.host(share.normed).astype(np.float64) @ w_gate.T                # the gate reads the norm's bf16 output
    idx, w, gap = O.route_grouped(logits, k, O.SIGMOID, groups, top_groups, O.GROUP_TOP2, 2.5, bias, 1)
    clear = gap > 1e-5 * (1 + np.abs(np.where(np.isfinite(bias), bias, 0)).max())
    assert clear.mean() > 0.9 and np.array_equal(H.host(share.idx)[clear], idx[clear])
    rows = O.pack_rows(*O.quantize_rows(v))
    ref = np.zeros((T, Hn))
    for e in range(E):
        t, j = np.nonzero(idx == e)
        if len(t):
            ref[t] += w[t, j, None] * O.expert_ffn(rows[t], Hn, [0, len(t)], [0], [experts[e]], act)
    if off:
        kept = H.host(share.slot_to_row).reshape(T, k) >= 0
        assert np.array_equal(kept, H.host(share.idx) >= 0)
    H.assert_close(y[clear], ref[clear], "bf16", (T, Hn, F, E))


@pytest.mark.parametrize("T,Hn,F,E,k", [(70, 512, 384, 16, 4), (300, 2048, 256, 64, 6), (64, 1024, 512, 130, 3)])
def test_share_in_a_graph_on_another_stream(T, Hn, F, E, k):
    r = np.random.default_rng(T + E)
    experts = experts_to_dev(make_experts(r, min(E, 64), Hn, F, O.ACT_SWIGLU)) if E <= 64 else experts_to_dev(make_experts(r, 2, Hn, F, O.ACT_SWIGLU)) * 32
    bias = np.where(np.arange(E) < 64, 0.0, -np.inf).astype(np.float32)        # of more than 64 experts the first 64 are here
    make = lambda: example().Fp8Share(T, Hn, F, E, k, O.ACT_SWIGLU, experts, H.dev(as_dtype(r.normal(size=(E, Hn)) * 0.05, "bf16"), "bf16"),  # noqa: E731
                                      torch.ones(Hn, dtype=torch.bfloat16, device=H.DEV), P.gate_rule(P.SCORE_SOFTMAX, 2, 2, P.GROUP_MAX), torch.from_numpy(bias).to(H.DEV))
    share = make()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    share.run(side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        share.run(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        share.x.normal_()
        share.residual.normal_()
        share.y.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (share.residual_out, share.rows, share.idx, share.w, share.y)]
        share.y.fill_(float("nan"))
        share.run(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (share.residual_out, share.rows, share.idx, share.w, share.y)))
        assert torch.isfinite(share.y.float()).all()


def test_example_runs(capsys):
    example().main(["--tokens", "300", "--hidden", "512", "--inner", "256", "--experts", "16", "--top", "2", "--groups", "4", "--top-groups", "2", "--steps", "2"])
    out = capsys.readouterr().out
    assert "finite: True" in out and "ffn" in out
