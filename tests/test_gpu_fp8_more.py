"""Further properties of the 8-bit share on the GPU: rounding of the norm, sizes beyond a launch.

Bounds.  The norm's v is formed in 64 bits from inputs that are exact there, so its error is a few 2^-52 (sums of at most 32768 terms: below
1e-12) and y is v rounded once: half a unit in the last place of its type, 2^(e - 24) in fp32 and 2^(e - 8) in bf16 for |v| in
[2^e, 2^(e + 1)).  Packed rows are v quantised, byte by byte: no v of these inputs lies within 1e-12 of the middle of two e4m3 numbers."""
import numpy as np
import pytest
import torch

from oracle import fp8_layer as O
from tests import harness as H
from tests.test_gpu_fp8 import as_dtype, compare_gate, run_norm

pytestmark = pytest.mark.gpu
P = H.P
DEV = H.DEV


# ------------------------------------------------------------------------------------------------ norm
def half_unit(v, dtype):
    return np.ldexp(1.0, np.floor(np.log2(np.maximum(np.abs(v), 1e-37))).astype(int) - (8 if dtype == "bf16" else 24))


@pytest.mark.parametrize("T,Hn,dtype,residual,gamma", [
    (1013, 1152, "fp32", False, True), (300, 128, "fp32", True, False), (64, 8192, "fp32", True, True), (9, 32768, "fp32", False, True),
    (500, 2048, "bf16", True, True), (33, 36, "fp32", False, True), (40, 1000, "bf16", False, True)])
def test_norm_rounds_once(T, Hn, dtype, residual, gamma):
    r = np.random.default_rng(T + Hn)
    x = as_dtype(r.normal(size=(T, Hn)) * 2.0 ** r.integers(-6, 7, (T, 1)), dtype)
    res = as_dtype(r.normal(size=(T, Hn)), dtype) if residual else None
    g = as_dtype(1 + 0.2 * r.normal(size=Hn), dtype) if gamma else None
    s = as_dtype(x.astype(np.float32) + res.astype(np.float32), dtype) if residual else x
    whole = Hn % 128 == 0
    _, y, rows = run_norm(x, res, g, 1e-6, dtype, want_rows=whole)
    v = O.norm(s, g, float(np.float32(1e-6)))                             # eps as the call takes it
    assert np.all(np.abs(y.double().numpy() - v) <= half_unit(v, dtype) + 1e-12 * np.abs(v))
    assert not whole or np.array_equal(rows.numpy(), O.pack_rows(*O.quantize_rows(v)))


def test_norm_of_rows_whose_squares_underflow_fp32():
    x = as_dtype(np.random.default_rng(8).normal(size=(5, 256)) * 1e-25, "fp32")
    _, y, _ = run_norm(x, None, None, 0.0, "fp32")
    v = O.norm(x, None, 0.0)
    assert np.all(np.abs(y.double().numpy() - v) <= half_unit(v, "fp32") + 1e-12 * np.abs(v))


def test_norm_values_below_and_above_the_range_of_fp32():
    # gamma of the largest and smallest numbers: v overflows to infinity, or underflows to zero and to fp32 subnormals
    x = np.ones((2, 256))
    g = np.where(np.arange(256) < 128, 3.0e38, 1e-38)
    x[:, 0] = 10.0
    _, y, rows = run_norm(x, None, g, 0.0, "fp32")
    v = O.norm(x, as_dtype(g, "fp32"), 0.0)
    assert np.all(np.isposinf(y[:, 0].numpy())) and np.all(rows[:, :128].numpy() == 0x7F)
    assert np.all(np.abs(y[:, 128:].double().numpy() - v[:, 128:]) <= 2.0 ** -150)
    assert np.array_equal(rows[:, 128:256].numpy(), O.quantize_rows(v[:, 128:])[0])


# ------------------------------------------------------------------------------------------------ more threads than a launch takes
def test_norm_of_more_rows_than_a_launch_has_threads_for():
    n, turns, Hn = 1 << 16, 1 << 10, 8                                       # 64 lanes per row: 2^32 threads, and five rows
    T = n * turns + 5
    r = np.random.default_rng(41)
    x = as_dtype(r.normal(size=(n, Hn)), "bf16")
    xd = H.dev(x, "bf16").repeat(turns + 1, 1)[:T].contiguous()
    y = torch.full_like(xd, float("nan"))
    P.moe_norm_fp8(xd, None, None, 1e-6, None, y, None)
    v = O.norm(x, None, float(np.float32(1e-6)))
    assert np.all(np.abs(y[:n].double().cpu().numpy() - v) <= half_unit(v, "bf16") + 1e-12 * np.abs(v))
    assert torch.equal(y[n:2 * n], y[:n]) and torch.equal(y[:n * turns].view(turns, -1)[1:], y[:n].view(1, -1).expand(turns - 1, -1)) and torch.equal(y[-5:], y[:5])


def test_gate_of_more_tokens_than_a_launch_has_threads_for():
    n, turns, Hn, E, k = 1 << 16, 1 << 13, 8, 4, 1                           # 8 lanes per token: 2^32 threads, and a block of tokens
    T = n * turns + 64
    r = np.random.default_rng(42)
    x, w = as_dtype(r.normal(size=(n, Hn)), "bf16"), as_dtype(r.normal(size=(E, Hn)) * 0.05, "bf16")
    xd = H.dev(x, "bf16").repeat(turns + 1, 1)[:T].contiguous()
    ctx = P.MoeCtx(T, Hn, E, k, 1, "bf16", 0)
    idx, wts = torch.full((T, k), -7, dtype=torch.int32, device=DEV), torch.full((T, k), float("nan"), device=DEV)
    ws = torch.empty(P.moe_route_grouped_workspace_bytes(ctx), dtype=torch.uint8, device=DEV)
    P.moe_route_grouped(ctx, xd, H.dev(w, "bf16"), P.gate_rule(O.SIGMOID), None, idx, wts, ws)
    compare_gate((idx[:n].cpu().numpy(), wts[:n].cpu().double().numpy()), x @ w.T, k, O.SIGMOID)
    for t in (idx, wts):
        assert torch.equal(t[:n * turns].view(turns, -1)[1:], t[:n].view(1, -1).expand(turns - 1, -1)) and torch.equal(t[-64:], t[:64])
    ctx.close()
