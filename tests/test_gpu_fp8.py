"""The 8-bit share on the GPU against the oracle in fp64: norm with packed rows, gate with groups, expert FFN on packed rows.

Tolerances.  A norm's v is formed in fp32 from a sum of H squares: its relative error is below 2e-6 for the sizes here (a tree
sum of at most 32768 terms, one square root, one division, two products).  A quantised value is right if it is a nearest e4m3 number of
some v within that; a scale byte if it is the definition's for some largest element within that.  fp32 y: 2e-6; bf16 y: half a
unit in the last place (2^(e - 8) for |v| in [2^e, 2^(e + 1))) beside it.  Gate weights: logits are fp32 sums of up to 4096 products of about 0.02, off by some 1e-6, which the scores
take over as relative errors of at most that size (softmax) or less: 1e-5.  Indices are compared where every gap that decides exceeds
1e-5 of the largest selection score.  FFN: the bounds of the bf16 FFN (one rounding of the output to bf16; an intermediate whose rounding
to 8 bits falls the other way, because the fp32 sum is 1.5e-5 off, is one in a thousand, 2^-4 off at most: 1e-3 of the norm)."""
import numpy as np
import pytest
import torch

from oracle import fp8_layer as O
from tests import harness as H

pytestmark = pytest.mark.gpu
P = H.P
DEV = H.DEV
V_ERR = 2e-6


def u8(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def as_dtype(v, dtype):
    """float64 host values on the grid of `dtype`."""
    t = torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(P.TORCH_DTYPE[dtype])
    return t.double().numpy()


# ------------------------------------------------------------------------------------------------ norm
def v_error(v, dtype):
    """Bound of |y - v|."""
    half_ulp = np.ldexp(1.0, np.floor(np.log2(np.maximum(np.abs(v), 1e-37))).astype(int) - 8) if dtype == "bf16" else 0.0
    return np.abs(v) * V_ERR + half_ulp * (1 + V_ERR) + 1e-37


def check_rows(rows, v):
    """Packed rows (host bytes) hold v quantised, up to V_ERR of v."""
    Hn = v.shape[1]
    q, b = O.unpack_rows(rows, Hn)
    assert not rows[:, Hn + Hn // 128:].any()                               # padding
    blocks = v.reshape(v.shape[0], -1, 128)
    amax = np.abs(blocks).max(2)
    bad = ~np.isfinite(amax)
    fine = np.where(bad, 0.0, amax)
    assert np.all((b == 127) | ~bad)
    assert np.all((O.scale_byte(fine * (1 - V_ERR)) <= b) & (b <= O.scale_byte(fine * (1 + V_ERR))) | bad)
    got = O.E4M3[q].reshape(blocks.shape)
    assert np.array_equal(np.isnan(got), np.broadcast_to(bad[..., None], got.shape))
    t = np.where(bad[..., None], 0.0, np.where(np.isfinite(blocks), blocks, 0.0) / np.ldexp(1.0, b.astype(int) - 127)[..., None])
    got = np.where(bad[..., None], 0.0, got)
    step = np.ldexp(1.0, np.maximum(np.floor(np.log2(np.maximum(np.abs(t), 1e-300))), -6).astype(int) - 3)
    assert np.all(np.abs(got - t) <= step / 2 + np.abs(t) * 2 * V_ERR)


def run_norm(x, residual, gamma, eps, dtype, want_out=True, want_y=True, want_rows=True):
    T, Hn = x.shape
    dt = P.TORCH_DTYPE[dtype]
    d = lambda a: None if a is None else H.dev(a, dtype)  # noqa: E731
    ro = torch.full((T, Hn), float("nan"), dtype=dt, device=DEV) if want_out else None
    y = torch.full((T, Hn), float("nan"), dtype=dt, device=DEV) if want_y else None
    rows = torch.full((T, P.moe_fp8_row_bytes(Hn)), 0xAA, dtype=torch.uint8, device=DEV) if want_rows else None
    P.moe_norm_fp8(d(x), d(residual), d(gamma), eps, ro, y, rows)
    torch.cuda.synchronize()
    return [None if t is None else t.cpu() for t in (ro, y, rows)]


@pytest.mark.parametrize("T,Hn,dtype,residual,gamma", [
    (1, 128, "bf16", True, True), (1, 128, "fp32", True, True), (3, 256, "bf16", False, True), (7, 1152, "fp32", True, True), (5, 1152, "bf16", True, False),
    (16, 4096, "bf16", True, True), (1013, 512, "bf16", True, True), (257, 640, "fp32", False, False), (9, 2048, "fp32", True, True), (4, 5120, "bf16", True, True),
    (3, 8192, "fp32", True, True), (2, 14336, "bf16", False, True), (3, 16512, "bf16", True, True), (2, 32768, "fp32", True, True)])
def test_norm(T, Hn, dtype, residual, gamma):
    r = np.random.default_rng(T * 7 + Hn)
    x = as_dtype(r.normal(size=(T, Hn)) * 2.0 ** r.integers(-6, 7, (T, 1)), dtype)
    x[:, r.integers(Hn, size=3)] *= 64.0
    x[T // 2] = 0.0                                                          # a row of zeros
    res = as_dtype(r.normal(size=(T, Hn)), dtype) if residual else None
    if res is not None:
        res[T // 2] = 0.0
    g = as_dtype(1 + 0.2 * r.normal(size=Hn), dtype) if gamma else None
    s = as_dtype((x.astype(np.float32) + res.astype(np.float32)), dtype) if residual else x
    ro, y, rows = run_norm(x, res, g, 1e-6, dtype)
    assert np.array_equal(ro.double().numpy(), s)
    v = O.norm(s, g, 1e-6)
    assert np.all(np.abs(y.double().numpy() - v) <= v_error(v, dtype))
    check_rows(rows.numpy(), v)


@pytest.mark.parametrize("Hn,dtype", [(8, "bf16"), (4, "fp32"), (36, "fp32"), (1000, "bf16"), (516, "fp32"), (4100, "fp32")])
def test_norm_of_widths_that_are_no_multiple_of_a_block(Hn, dtype):
    r = np.random.default_rng(Hn)
    x, res = as_dtype(r.normal(size=(5, Hn)), dtype), as_dtype(r.normal(size=(5, Hn)), dtype)
    g = as_dtype(r.normal(size=Hn), dtype)
    s = as_dtype(x.astype(np.float32) + res.astype(np.float32), dtype)
    ro, y, _ = run_norm(x, res, g, 1e-5, dtype, want_rows=False)
    v = O.norm(s, g, 1e-5)
    assert np.array_equal(ro.double().numpy(), s)
    assert np.all(np.abs(y.double().numpy() - v) <= v_error(v, dtype))


def test_norm_quantises_exactly_where_the_arithmetic_is_exact():
    # rows of +-1 with eps = 0 have the norm 1, so v = gamma: powers of two, values halfway between e4m3 numbers, block maxima at the limit of a scale
    r = np.random.default_rng(5)
    x = np.where(r.random((4, 512)) < 0.5, -1.0, 1.0)
    g = np.concatenate([2.0 ** r.integers(-20, 5, 128), r.integers(1, 449, 128), np.where(np.arange(128) == 5, 448.0, 17.0), np.where(np.arange(128) == 9, 449.0, 9.0 + 2.0 ** -3)])
    _, y, rows = run_norm(x, None, g, 0.0, "fp32")
    assert np.array_equal(y.double().numpy(), x * g)
    assert np.array_equal(rows.numpy(), O.pack_rows(*O.quantize_rows(x * g)))


def test_norm_rows_with_infinities_and_nans_stay_by_themselves():
    x = np.random.default_rng(6).normal(size=(6, 256))
    clean = run_norm(x, None, None, 1e-6, "fp32")
    x[1, 7], x[3, 200], x[4] = np.inf, np.nan, 3e38                          # an infinite sum of squares: zeros, not NaN
    _, y, rows = run_norm(x, None, None, 1e-6, "fp32")
    for t in (0, 2, 5):
        assert torch.equal(y[t], clean[1][t]) and torch.equal(rows[t], clean[2][t])
    q, b = O.unpack_rows(rows.numpy(), 256)
    assert np.all(q[3] == 0x7F) and np.all(b[3] == 127)                      # NaN in the sum: the whole row
    assert np.all(q[1, :128] == 0x7F) and np.all(O.E4M3[q[1, 128:]] == 0)    # inf * 0 in its block, zeros in the other
    assert np.all(O.E4M3[q[4]] == 0)


def test_norm_in_place_and_with_each_output_alone():
    r = np.random.default_rng(7)
    x, res = as_dtype(r.normal(size=(33, 1024)), "bf16"), as_dtype(r.normal(size=(33, 1024)), "bf16")
    ro, y, rows = run_norm(x, res, None, 1e-6, "bf16")
    for one in range(3):
        got = run_norm(x, res, None, 1e-6, "bf16", *(i == one for i in range(3)))
        assert torch.equal(got[one].view(torch.uint8), (ro, y, rows)[one].view(torch.uint8))
    xd, rd = H.dev(x, "bf16"), H.dev(res, "bf16")
    P.moe_norm_fp8(xd, rd, None, 1e-6, rd, xd, None)
    torch.cuda.synchronize()
    assert torch.equal(rd.cpu(), ro) and torch.equal(xd.cpu(), y)


def test_norm_binding_checks_shapes():
    x = torch.zeros(4, 256, device=DEV)
    with pytest.raises(ValueError):
        P.moe_norm_fp8(x, None, None, 1e-6, None, torch.zeros(4, 128, device=DEV), None)
    with pytest.raises(ValueError):
        P.moe_norm_fp8(x, None, None, 1e-6, None, None, torch.zeros(4, 300, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        P.moe_norm_fp8(x, None, torch.zeros(256, dtype=torch.bfloat16, device=DEV), 1e-6, None, x, None)
    with pytest.raises(ValueError):
        P.moe_norm_fp8(x.t(), None, None, 1e-6, None, x.t(), None)


# ------------------------------------------------------------------------------------------------ gate
def run_gate(x, w, k, dtype, score, n_groups=1, top_groups=1, group_rank=0, scale=1.0, bias=None, renorm=0):
    T, Hn = x.shape
    E = w.shape[0]
    ctx = P.MoeCtx(T, Hn, E, k, 1, dtype, renorm)
    idx = torch.full((T, k), -7, dtype=torch.int32, device=DEV)
    wts = torch.full((T, k), float("nan"), dtype=torch.float32, device=DEV)
    ws = torch.full((P.moe_route_grouped_workspace_bytes(ctx),), 0xFF, dtype=torch.uint8, device=DEV)
    b = None if bias is None else torch.from_numpy(np.asarray(bias, dtype=np.float32)).to(DEV)
    P.moe_route_grouped(ctx, H.dev(x, dtype), H.dev(w, dtype), P.gate_rule(score, n_groups, top_groups, group_rank, scale), b, idx, wts, ws)
    torch.cuda.synchronize()
    ctx.close()
    return idx.cpu().numpy(), wts.cpu().double().numpy()


def gate_inputs(T, Hn, E, dtype, seed):
    r = np.random.default_rng(seed)
    return as_dtype(r.normal(size=(T, Hn)), dtype), as_dtype(r.normal(size=(E, Hn)) * 0.05, dtype), r


def compare_gate(got, logits, k, score, bias=None, **rule):
    idx, w = got
    ref_idx, ref_w, gap = O.route_grouped(logits, k, score, bias=bias, **rule)
    c, _ = O.selection(logits, score, bias)
    clear = gap > 1e-5 * np.abs(np.where(np.isfinite(c), c, 0.0)).max(1)
    assert clear.mean() > 0.9 or len(clear) < 20
    assert np.array_equal(idx[clear], ref_idx[clear])
    assert np.all(np.abs(w - ref_w)[clear] <= 1e-5 * np.abs(ref_w[clear]) + 1e-30)


@pytest.mark.parametrize("T,Hn,E,k,dtype,score,n_groups,top_groups,group_rank,bias,renorm,scale", [
    (1, 256, 8, 2, "bf16", O.SOFTMAX, 1, 1, 0, False, 0, 1.0),
    (1, 64, 1, 1, "fp32", O.SIGMOID, 1, 1, 1, True, 1, 1.0),
    (64, 2048, 64, 6, "bf16", O.SOFTMAX, 8, 3, 0, False, 0, 2.5),
    (65, 2048, 64, 6, "bf16", O.SIGMOID, 8, 4, 1, True, 1, 1.0),
    (130, 1024, 256, 8, "bf16", O.SIGMOID, 8, 4, 1, True, 1, 2.5),
    (33, 512, 256, 16, "fp32", O.SOFTMAX, 16, 5, 1, True, 1, 1.0),
    (77, 1152, 24, 3, "fp32", O.SIGMOID, 6, 4, 1, True, 1, 1.0),
    (77, 1152, 24, 3, "bf16", O.SOFTMAX, 6, 2, 0, True, 0, 1.0),
    (19, 72, 7, 7, "bf16", O.SOFTMAX, 7, 7, 1, False, 1, 1.0),               # k = E, H no multiple of 32, groups of one
    (20, 36, 130, 5, "fp32", O.SIGMOID, 10, 3, 1, True, 1, -1.0),
    (31, 8, 200, 4, "bf16", O.SIGMOID, 40, 9, 1, True, 0, 1.0),
    (50, 4096, 255, 1, "bf16", O.SOFTMAX, 5, 1, 0, True, 1, 1.0),
    (600, 256, 96, 4, "bf16", O.SIGMOID, 3, 2, 1, True, 1, 1.0),
    (3, 128, 256, 2, "fp32", O.SOFTMAX, 256, 9, 1, False, 0, 1.0)])
def test_gate(T, Hn, E, k, dtype, score, n_groups, top_groups, group_rank, bias, renorm, scale):
    x, w, r = gate_inputs(T, Hn, E, dtype, T + Hn + E)
    b = (r.normal(size=E) * 0.1).astype(np.float32) if bias else None
    rule = dict(n_groups=n_groups, top_groups=top_groups, group_rank=group_rank, scale=scale, renorm=renorm)
    compare_gate(run_gate(x, w, k, dtype, score, bias=b, **rule), x @ w.T, k, score, bias=b, **rule)


@pytest.mark.parametrize("T,Hn,E,k,dtype,n_groups,top_groups", [
    (1, 1024, 16, 2, "bf16", 4, 2), (515, 1024, 16, 2, "bf16", 4, 2), (5000, 512, 16, 3, "fp32", 4, 2), (4096, 512, 64, 6, "bf16", 8, 4), (40, 768, 32, 4, "bf16", 8, 3),      # one kernel
    (4097, 512, 64, 6, "bf16", 8, 4), (40, 4096, 8, 2, "bf16", 2, 1), (1100, 2048, 16, 2, "bf16", 4, 2), (130, 1024, 32, 4, "fp32", 8, 3),                                 # two
    (12300, 256, 64, 6, "bf16", 8, 4), (12289, 128, 96, 4, "fp32", 3, 2)])                                                                                                   # one, of 64 tokens per block
def test_gate_in_one_kernel_and_in_two(T, Hn, E, k, dtype, n_groups, top_groups):
    x, w, r = gate_inputs(T, Hn, E, dtype, T + E)
    b = (r.normal(size=E) * 0.1).astype(np.float32)
    rule = dict(n_groups=n_groups, top_groups=top_groups, group_rank=O.GROUP_TOP2, scale=2.5, renorm=1)
    compare_gate(run_gate(x, w, k, dtype, O.SIGMOID, bias=b, **rule), x @ w.T, k, O.SIGMOID, bias=b, **rule)


@pytest.mark.parametrize("E,k,n_groups,top_groups", [(8, 4, 1, 1), (64, 6, 8, 3), (200, 16, 8, 8), (256, 16, 16, 4)])
def test_gate_equal_scores_go_to_the_lower_index(E, k, n_groups, top_groups):
    x, w, r = gate_inputs(40, 256, E, "bf16", E)
    w = w[r.integers(0, max(2, E // 8), E)]                                  # every row several times: equal logits, bit for bit
    x[3] = 0.0                                                               # all equal
    for score in (O.SOFTMAX, O.SIGMOID):
        for rank in (O.GROUP_MAX, O.GROUP_TOP2):
            rule = dict(n_groups=n_groups, top_groups=top_groups, group_rank=rank)
            logits = (x @ w.T).astype(np.float32).astype(np.float64)         # duplicated rows stay equal in any arithmetic
            idx, _ = run_gate(x, w, k, "bf16", score, **rule)
            ref, _, _ = O.route_grouped(np.round(logits, 4), k, score, **rule)
            clean = [t for t in range(40) if np.diff(np.unique(logits[t])).min(initial=1.0) > 1e-3]
            assert 3 in clean and np.array_equal(idx[clean], ref[clean])


def test_gate_experts_out_of_service():
    x, w, r = gate_inputs(50, 256, 24, "bf16", 3)
    logits = x @ w.T
    for off in ([0], [4, 5, 6, 7], list(range(1, 24)), list(range(24)), [0, 1, 2, 8, 9, 10, 16]):
        b = np.zeros(24, dtype=np.float32)
        b[off] = -np.inf
        for rank in (0, 1):
            for renorm in (0, 1):
                rule = dict(n_groups=6, top_groups=2, group_rank=rank, renorm=renorm)
                got = run_gate(x, w, 3, "bf16", O.SIGMOID, bias=b, **rule)
                compare_gate(got, logits, 3, O.SIGMOID, bias=b, **rule)
                assert not np.isin(got[0], off).any() and np.all(got[1][got[0] < 0] == 0)
    b = np.full(24, np.finfo(np.float32).min, dtype=np.float32)              # the type's lowest value is no minus infinity
    idx, _ = run_gate(x, w, 3, "bf16", O.SIGMOID, bias=b)
    assert np.array_equal(idx, np.tile([0, 1, 2], (50, 1)))                  # every score is lost beside it: equal
    b = np.where(np.arange(24) == 9, np.nan, 0.0).astype(np.float32)         # NaN: never chosen
    got = run_gate(x, w, 3, "bf16", O.SOFTMAX, bias=b)
    compare_gate(got, logits, 3, O.SOFTMAX, bias=b)
    assert not (got[0] == 9).any()


def test_gate_tokens_that_are_not_finite_stay_by_themselves():
    x, w, _ = gate_inputs(40, 128, 16, "fp32", 9)
    clean = run_gate(x, w, 2, "fp32", O.SOFTMAX, renorm=1)
    x[5, 3], x[17] = np.nan, np.inf
    for score in (O.SOFTMAX, O.SIGMOID):
        clean = run_gate(np.nan_to_num(x, posinf=0.0), w, 2, "fp32", score, renorm=1)
        idx, wts = run_gate(x, w, 2, "fp32", score, renorm=1)
        rest = [t for t in range(40) if t not in (5, 17)]
        assert np.array_equal(idx[rest], clean[0][rest]) and np.array_equal(wts[rest], clean[1][rest])
        assert np.all(idx[5] == -1) and np.all(wts[5] == 0)                  # all scores NaN: nothing is chosen


def test_gate_scores_that_vanish():
    # sigmoid(-2e4) is 0 for every expert: equal scores, and a sum of 0 gives weights of 0, not NaN
    x = np.ones((3, 128))
    idx, w = run_gate(x, np.full((8, 128), -160.0), 2, "fp32", O.SIGMOID, renorm=1)
    assert np.array_equal(idx, np.tile([0, 1], (3, 1))) and np.all(w == 0)
    # logits of +-2e4: the softmax is one-hot, nothing overflows
    wg = np.full((8, 128), -160.0)
    wg[5] = 160.0
    idx, w = run_gate(x, wg, 2, "fp32", O.SOFTMAX, renorm=0)
    assert np.array_equal(idx, np.tile([5, 0], (3, 1))) and np.array_equal(w, np.tile([1.0, 0.0], (3, 1)))


def test_gate_refusals():
    ctx = P.MoeCtx(4, 128, 24, 3, 1, "bf16", 0)
    x, w = torch.zeros(4, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(24, 128, dtype=torch.bfloat16, device=DEV)
    idx, wt = torch.zeros(4, 3, dtype=torch.int32, device=DEV), torch.zeros(4, 3, device=DEV)
    ws = torch.zeros(P.moe_route_grouped_workspace_bytes(ctx), dtype=torch.uint8, device=DEV)
    for want, rule in (("MOE_EINVAL", (2,)), ("MOE_EINVAL", (0, 6, 2, 2)), ("MOE_EINVAL", (0, 0, 1)), ("MOE_EINVAL", (0, 6, 0)), ("MOE_ESHAPE", (0, 5, 2)),
                       ("MOE_ESHAPE", (0, 6, 7)), ("MOE_ESHAPE", (0, 12, 1)), ("MOE_EINVAL", (0, 1, 1, 0, float("nan"))), ("MOE_EINVAL", (0, 1, 1, 0, float("inf")))):
        with pytest.raises(P.MoeError) as ei:
            P.moe_route_grouped(ctx, x, w, P.gate_rule(*rule), None, idx, wt, ws)
        assert ei.value.name == want, rule
    for want, args in (("MOE_EINVAL", (None, w, P.gate_rule(), None, idx, wt, ws)), ("MOE_EINVAL", (x, w, P.gate_rule(), None, None, wt, ws)),
                       ("MOE_ESHAPE", (x, w, P.gate_rule(), None, idx, wt, ws[:16])), ("MOE_EALIGN", (x, w, P.gate_rule(), None, idx, wt, ws[16:]))):
        with pytest.raises(P.MoeError) as ei:
            P.moe_route_grouped(ctx, *args)
        assert ei.value.name == want
    assert P.moe_route_grouped_workspace_bytes(ctx) >= 256


def test_gate_drops_rank_reuse():
    # a grouped gate between moe_traffic and moe_dispatch has new indices: the ranks of the old ones must not be used
    T, E, k = 64, 8, 2
    ctx = P.MoeCtx(T, 128, E, k, 1, "bf16", 0)
    ctx.set_rank_reuse(True)
    x, w, r = gate_inputs(T, 128, E, "bf16", 1)
    xd, wd = H.dev(x, "bf16"), H.dev(w, "bf16")
    i32 = dict(dtype=torch.int32, device=DEV)
    idx, wt = torch.zeros(T, k, **i32), torch.zeros(T, k, device=DEV)
    ws = torch.zeros(P.moe_route_grouped_workspace_bytes(ctx), dtype=torch.uint8, device=DEV)
    P.moe_traffic(ctx, idx, [0] * E, torch.zeros(E, **i32), torch.zeros(1, **i32), torch.zeros(1, **i32))
    P.moe_route_grouped(ctx, xd, wd, P.gate_rule(), None, idx, wt, ws)
    send = torch.zeros(T * k, 128, dtype=torch.bfloat16, device=DEV)
    s2r, r2s, so, se = torch.zeros(T * k, **i32), torch.zeros(T * k, **i32), torch.zeros(E + 1, **i32), torch.zeros(E, **i32)
    P.moe_dispatch(ctx, xd, idx, [0] * E, [0], send, s2r, r2s, so, se)
    torch.cuda.synchronize()
    assert sorted(s2r.tolist()) == list(range(T * k))


# ------------------------------------------------------------------------------------------------ FFN
def make_experts(r, n, Hn, F, act):
    out = []
    for _ in range(n):
        e = {}
        for name, shape in (("1", (F, Hn)), ("_up", (F, Hn)), ("_down", (Hn, F))):
            if name == "_up" and act != O.ACT_SWIGLU:
                e["w_up"] = e["s_up"] = None
                continue
            w = r.normal(size=shape) * 0.05 * 2.0 ** np.repeat(np.repeat(r.integers(-3, 4, (shape[0] // 128, shape[1] // 128)), 128, 0), 128, 1)
            e["w" + name], e["s" + name] = O.quantize_weight(w)
        out.append(e)
    return out


def experts_to_dev(experts):
    return [{k: None if v is None else u8(v) for k, v in e.items()} for e in experts]


def make_rows(r, R, Hn):
    return O.pack_rows(*O.quantize_rows(r.normal(size=(R, Hn)) * 2.0 ** r.integers(-8, 9, (R, 1)) * 0.05))


def run_ffn8(rows, seg_offset, seg_expert, experts_dev, Hn, F, act, stream=None):
    R = rows.shape[0]
    so = torch.tensor(np.asarray(seg_offset, dtype=np.int32), device=DEV)
    se = torch.tensor(np.asarray(seg_expert, dtype=np.int32), device=DEV)
    ws = torch.full((max(P.moe_ffn_fp8_workspace_bytes(R, Hn, F, act), 256),), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full((R, Hn), float("nan"), dtype=torch.bfloat16, device=DEV)
    P.moe_expert_ffn_fp8(u8(rows), R, so, se, len(seg_expert), experts_dev, Hn, F, act, out, ws)
    torch.cuda.synchronize()
    return out


def check_ffn(rows, so, se, experts, Hn, F, act):
    out = H.host(run_ffn8(rows, so, se, experts_to_dev(experts), Hn, F, act)).astype(np.float64)
    ref = O.expert_ffn(rows, Hn, so, se, experts, act)
    assert np.array_equal(np.isnan(out), np.isnan(ref))                      # rows outside every segment stay as they were
    used = ~np.isnan(ref[:, 0])
    # row by row scales differ by powers of two: compare every row against its own size
    size = np.sqrt(np.mean(ref[used] ** 2, axis=1, keepdims=True)) + 1e-30
    H.assert_close(out[used] / size, ref[used] / size, "bf16", (len(rows), Hn, F, act))


@pytest.mark.parametrize("act", [O.ACT_SILU_MLP, O.ACT_GELU_MLP, O.ACT_SWIGLU])
@pytest.mark.parametrize("R,Hn,F", [(1, 128, 128), (2, 256, 128), (17, 128, 384), (33, 384, 640), (64, 256, 256), (65, 1152, 256), (129, 256, 1408), (300, 640, 512)])
def test_ffn_one_expert(R, Hn, F, act):
    r = np.random.default_rng(R + Hn + F + act)
    check_ffn(make_rows(r, R, Hn), [0, R], [0], make_experts(r, 1, Hn, F, act), Hn, F, act)


@pytest.mark.parametrize("seg_rows,seg_expert,n_local", [
    ([0, 5, 0, 1], [0, 1, 2, 1], 3),                                         # empty segments
    ([3] * 24, [i % 4 for i in range(24)], 4),                               # gathered rows of many short segments
    ([40, 90, 1, 70, 33], [2, 0, 2, 0, 1], 4),                               # an expert without rows
    ([7, 9, 11], [0, 9, -1], 2),                                             # experts that do not exist
    ([2] * 130, [(i * 5) % 7 for i in range(130)], 7),                       # more than 64 segments
    ([257, 300], [1, 0], 2),
    ([2] * 699 + [13], [i % 4 for i in range(700)], 4)])                      # tile maps of two heights do not fit beside each other
def test_ffn_segments(seg_rows, seg_expert, n_local):
    r = np.random.default_rng(len(seg_rows))
    Hn, F, act = 256, 384, O.ACT_SWIGLU
    so = np.concatenate([[3], 3 + np.cumsum(seg_rows)])                      # three rows in front and two behind belong to no segment
    rows = make_rows(r, int(so[-1]) + 2, Hn)
    check_ffn(rows, so, seg_expert, make_experts(r, n_local, Hn, F, act), Hn, F, act)


@pytest.mark.parametrize("R,Hn,F,act,n_local,nseg", [(403, 2048, 1408, O.ACT_SWIGLU, 4, 64), (37, 1024, 2304, O.ACT_SWIGLU, 1, 8), (700, 1152, 2304, O.ACT_SILU_MLP, 4, 24),
                                                     (1500, 1024, 1024, O.ACT_GELU_MLP, 3, 12), (90, 2048, 1408, O.ACT_SWIGLU, 8, 16), (2200, 512, 640, O.ACT_SWIGLU, 2, 4)])
def test_ffn_of_ordinary_sizes(R, Hn, F, act, n_local, nseg):
    r = np.random.default_rng(R)
    so = np.concatenate([[0], np.sort(r.integers(0, R + 1, nseg - 1)), [R]])
    check_ffn(make_rows(r, R, Hn), so, r.integers(0, n_local, nseg), make_experts(r, n_local, Hn, F, act), Hn, F, act)


def plan_of(R, n_used, nseg, Hn, F, act):
    import ctypes as C
    from paper_2410_17043_amd import _lib
    p = (C.c_int32 * 5)()
    assert _lib.load().moe_selfcheck_fp8_plan(R, n_used, nseg, Hn, F, act, 256, p) == 0
    return dict(zip(("mt", "bm1", "bm2", "deep", "pieces"), p))


@pytest.mark.parametrize("R,Hn,F,act,n_local,want", [
    (5, 1024, 8192, O.ACT_SWIGLU, 1, dict(mt=1)), (20, 1024, 8192, O.ACT_GELU_MLP, 1, dict(mt=2)), (60, 896, 8064, O.ACT_SWIGLU, 1, dict(mt=4)),
    (100, 256, 4096, O.ACT_SILU_MLP, 2, dict(mt=4, pieces=8)),
    (1100, 128, 14336, O.ACT_GELU_MLP, 1, dict(mt=0, bm2=256, pieces=7)), (1300, 384, 8192, O.ACT_SWIGLU, 2, dict(mt=0, bm2=256, pieces=8)),
    (1200, 512, 640, O.ACT_SWIGLU, 3, dict(mt=0, bm1=64, bm2=128, deep=1)), (9000, 384, 1408, O.ACT_SWIGLU, 2, dict(mt=0, bm1=256)),
    (9000, 256, 2304, O.ACT_SILU_MLP, 2, dict(mt=0, bm1=128)), (3000, 512, 1408, O.ACT_SWIGLU, 1, dict(mt=0, bm2=128))])
def test_ffn_by_each_kernel(R, Hn, F, act, n_local, want):
    r = np.random.default_rng(R + F)
    so = [R * i // n_local for i in range(n_local + 1)]
    plan = plan_of(R, n_local, n_local, Hn, F, act)
    assert {k: plan[k] for k in want} == want, plan
    check_ffn(make_rows(r, R, Hn), so, list(range(n_local)), make_experts(r, n_local, Hn, F, act), Hn, F, act)


def test_ffn_rows_do_not_depend_on_others():
    r = np.random.default_rng(11)
    Hn, F, act, R = 512, 640, O.ACT_SWIGLU, 300
    rows, experts = make_rows(r, R, Hn), experts_to_dev(make_experts(r, 2, Hn, F, act))
    clean = run_ffn8(rows, [0, 140, R], [0, 1], experts, Hn, F, act)
    rows2 = rows.copy()
    rows2[5, :128], rows2[200, 17] = 0x7F, 0xFF                              # rows that hold NaN
    got = run_ffn8(rows2, [0, 140, R], [0, 1], experts, Hn, F, act)
    assert torch.isnan(got[5]).all() and torch.isnan(got[200]).all()
    keep = [t for t in range(R) if t not in (5, 200)]
    assert torch.equal(got[keep], clean[keep])


def test_ffn_intermediate_that_overflows_is_nan_for_its_row_only():
    r = np.random.default_rng(12)
    Hn, F, act = 128, 128, O.ACT_SWIGLU
    e = make_experts(r, 1, Hn, F, act)
    for n in ("s1", "s_up"):
        e[0][n][:] = 240                                                     # products beyond the range of fp32 for large rows
    rows = make_rows(r, 8, Hn)
    rows[3, 128] = 200
    out = run_ffn8(rows, [0, 8], [0], experts_to_dev(e), Hn, F, act)
    assert torch.isnan(out[3]).all()


def test_ffn_zero_rows_and_zero_weights():
    r = np.random.default_rng(13)
    Hn, F, act = 256, 256, O.ACT_GELU_MLP
    e = make_experts(r, 1, Hn, F, act)
    rows = make_rows(r, 70, Hn)
    rows[10] = O.pack_rows(*O.quantize_rows(np.zeros((1, Hn))))[0]
    out = run_ffn8(rows, [0, 70], [0], experts_to_dev(e), Hn, F, act)
    assert torch.all(out[10] == 0) and not torch.isnan(out).any()
    e[0]["w_down"][:] = 0
    assert torch.all(run_ffn8(rows, [0, 70], [0], experts_to_dev(e), Hn, F, act) == 0)


def test_ffn_runs_twice_alike_and_in_a_graph_on_another_stream():
    r = np.random.default_rng(14)
    Hn, F, act, R = 1024, 768, O.ACT_SWIGLU, 500
    experts = experts_to_dev(make_experts(r, 3, Hn, F, act))
    so = torch.tensor([0, 100, 333, 400, R], dtype=torch.int32, device=DEV)
    se = torch.tensor([0, 2, 0, 1], dtype=torch.int32, device=DEV)
    recv = u8(make_rows(r, R, Hn))
    ws = torch.full((P.moe_ffn_fp8_workspace_bytes(R, Hn, F, act),), 0xFF, dtype=torch.uint8, device=DEV)
    outs = [torch.full((R, Hn), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(3)]
    for o in outs[:2]:
        P.moe_expert_ffn_fp8(recv, R, so, se, 4, experts, Hn, F, act, o, ws)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and not torch.isnan(outs[0]).any()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        call = P.bind_expert_ffn_fp8(recv, R, so, se, 4, experts, Hn, F, act, outs[2], ws)
        call()
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            call(torch.cuda.current_stream().cuda_stream)
    fresh = make_rows(r, R, Hn)
    for rows in (fresh, make_rows(r, R, Hn), fresh):
        recv.copy_(u8(rows))
        torch.cuda.synchronize()
        outs[2].fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        P.moe_expert_ffn_fp8(recv, R, so, se, 4, experts, Hn, F, act, outs[0], ws)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2])


# ------------------------------------------------------------------------------------------------ arrays beyond 4 GiB
def every_turn_alike(t, n):
    """The rows of t repeat with period n, bit for bit."""
    raw = t.view(torch.uint8).reshape(t.shape[0], -1)
    return all(torch.equal(raw[i:i + n], raw[:min(n, t.shape[0] - i)]) for i in range(n, t.shape[0], n))


def test_norm_and_gate_beyond_4_gib():
    n, turns, Hn, E, k = 4096, 130, 4096, 16, 2
    T = n * turns
    assert T * Hn * 2 > 2 ** 32
    r = np.random.default_rng(31)
    x, g = as_dtype(r.normal(size=(n, Hn)), "bf16"), as_dtype(1 + 0.2 * r.normal(size=Hn), "bf16")
    xd = H.dev(x, "bf16").repeat(turns, 1)
    y = torch.empty_like(xd)
    rows = torch.empty(T, P.moe_fp8_row_bytes(Hn), dtype=torch.uint8, device=DEV)
    P.moe_norm_fp8(xd, None, H.dev(g, "bf16"), 1e-6, None, y, rows)
    some = [0, 1, 2047, n - 1]
    v = O.norm(x[some], g, 1e-6)
    assert np.all(np.abs(y[some].double().cpu().numpy() - v) <= v_error(v, "bf16"))
    check_rows(rows[some].cpu().numpy(), v)
    assert every_turn_alike(y, n) and every_turn_alike(rows, n)
    del y, rows
    w = as_dtype(r.normal(size=(E, Hn)) * 0.05, "bf16")
    ctx = P.MoeCtx(T, Hn, E, k, 1, "bf16", 1)
    idx, wts = torch.full((T, k), -7, dtype=torch.int32, device=DEV), torch.zeros(T, k, device=DEV)
    ws = torch.empty(P.moe_route_grouped_workspace_bytes(ctx), dtype=torch.uint8, device=DEV)
    P.moe_route_grouped(ctx, xd, H.dev(w, "bf16"), P.gate_rule(O.SIGMOID), None, idx, wts, ws)
    compare_gate((idx[:n].cpu().numpy(), wts[:n].cpu().double().numpy()), x @ w.T, k, O.SIGMOID, renorm=1)
    assert every_turn_alike(idx, n) and every_turn_alike(wts, n)
    ctx.close()


def test_ffn_beyond_4_gib():
    n, R, Hn, F, act = 8192, 560000, 7680, 128, O.ACT_SILU_MLP
    pitch = P.moe_fp8_row_bytes(Hn)
    assert R * pitch > 2 ** 32                                               # rows are no longer gathered: tiles of adjacent rows only
    r = np.random.default_rng(32)
    base, experts = make_rows(r, n, Hn), make_experts(r, 2, Hn, F, act)
    recv = u8(base).repeat(-(-R // n), 1)[:R]
    so, se = [0, 200001, 400003, R], [1, 0, 1]
    out = torch.full((R, Hn), float("nan"), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(P.moe_ffn_fp8_workspace_bytes(R, Hn, F, act), dtype=torch.uint8, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    P.moe_expert_ffn_fp8(recv, R, torch.tensor(so, **i32), torch.tensor(se, **i32), 3, experts_to_dev(experts), Hn, F, act, out, ws)
    for owner, some in ((1, [0, 1, n - 1, 200000, 400003, 2 ** 32 // pitch, 2 ** 32 // pitch + 1, R - 1]), (0, [200001, 2 ** 32 // (2 * Hn), 2 ** 32 // (2 * Hn) + 1, 400002])):
        got = out[some].double().cpu().numpy()
        ref = O.expert_ffn(base[[i % n for i in some]], Hn, [0, len(some)], [owner], experts, act)
        size = np.sqrt(np.mean(ref ** 2, axis=1, keepdims=True))
        H.assert_close(got / size, ref / size, "bf16", (owner,))
    assert every_turn_alike(out[:200001], n) and every_turn_alike(out[200001:400003], n) and every_turn_alike(out[400003:], n)
