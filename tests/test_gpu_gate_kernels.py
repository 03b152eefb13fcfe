"""Every kernel that the gate with groups can run, against the oracle: (tokens per block, experts, one kernel or two, type), rows whose last 128 bytes are
partly beyond them, the most groups.  Bounds as in test_gpu_fp8."""
import numpy as np
import pytest
import torch

from oracle import fp8_layer as O
from tests.test_fp8_plans import gate_plan
from tests.test_gpu_fp8 import compare_gate, gate_inputs, run_gate

pytestmark = pytest.mark.gpu

# T, H in bytes / 16, E, k, groups, kept groups, plan: tokens per block and whether one kernel does it all
CASES = [
    (40, 33, 12, 3, 4, 2, 16, True), (40, 33, 28, 4, 7, 3, 16, True), (77, 33, 60, 6, 6, 4, 16, True),                                   # gate_logits_kernel
    (40, 257, 12, 3, 4, 2, 16, False), (200, 257, 28, 4, 7, 3, 16, False), (1000, 161, 60, 6, 6, 4, 16, False),
    (70, 137, 100, 6, 10, 4, 16, False), (600, 137, 200, 8, 8, 4, 16, False), (33, 137, 256, 16, 256, 40, 16, False),                    # gate_logits_wide_kernel
    (1030, 257, 28, 4, 7, 3, 64, False), (1030, 161, 60, 6, 6, 4, 64, False), (1030, 137, 100, 6, 10, 4, 64, False),
    (1030, 137, 256, 8, 8, 4, 64, False), (3000, 41, 200, 8, 200, 40, 64, False),
    (12300, 9, 20, 3, 5, 2, 64, True), (12289, 17, 60, 6, 6, 4, 64, True), (12300, 9, 100, 6, 10, 4, 64, True),
    (12289, 9, 200, 8, 8, 4, 64, True), (12300, 17, 256, 16, 256, 40, 64, True)]


def test_the_cases_reach_every_kernel():
    wide = [(tokens, next(e for e in (32, 64, 128, 256) if E <= e), one) for _, _, E, _, _, _, tokens, one in CASES if tokens == 64 or E > 64]
    assert set(wide) == {(16, 128, False), (16, 256, False)} | {(64, e, one) for e in (32, 64, 128, 256) for one in (False, True)}
    assert {(-(-E // 16), one) for _, _, E, _, _, _, tokens, one in CASES if tokens == 16 and E <= 64} == {(n, one) for n in (1, 2, 4) for one in (False, True)}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,units,E,k,n_groups,top_groups,tokens,one", CASES)
def test_gate_by_each_kernel(T, units, E, k, n_groups, top_groups, tokens, one, dtype):
    Hn = units * (8 if dtype == "bf16" else 4)
    assert units % 8 != 0                                                    # the last step is partly beyond the row
    plan = gate_plan(T, Hn, E, n_groups, dtype)
    assert (plan["tokens"], plan["pieces"] == 0) == (tokens, one), plan
    n = min(T, 400)                                                          # tokens that differ
    x, w, r = gate_inputs(n, Hn, E, dtype, T + Hn + E)
    b = (r.normal(size=E) * 0.1).astype(np.float32)
    b[int(r.integers(E))] = -np.inf
    turns = np.arange(T) % n
    for score, rank, renorm in ((O.SIGMOID, O.GROUP_TOP2, 1), (O.SOFTMAX, O.GROUP_MAX, 0)):
        rule = dict(n_groups=n_groups, top_groups=top_groups, group_rank=rank, scale=2.5, renorm=renorm)
        idx, wts = run_gate(x[turns], w, k, dtype, score, bias=b, **rule)
        compare_gate((idx[:n], wts[:n]), x @ w.T, k, score, bias=b, **rule)
        assert np.array_equal(idx, idx[turns]) and np.array_equal(wts, wts[turns])   # wherever a token stands
