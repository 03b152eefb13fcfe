"""Integer rows and the experts' FFN on them, on the GPU.

Bit for bit, with rows and first weights that are not negative: sums are exact whole numbers, the activations return a large argument itself (sigmoid is 1 from 17 on in
fp32; tanh likewise), and what is left are the roundings that the definition names (fp32 products with the scales, bf16, whole numbers), which numpy's float32 makes alike.  A
product that is lost, a scale of another row or column, a cut, a tie that goes the wrong way change it.

With weights of both signs against the oracle in 64 bits: the activations are off by some 1e-6 then, which one element of h in a thousand takes to the neighbouring bf16 number
(2^-8 of it); where that is a row's largest, the row is quantised anew, which moves it by about 1/127 / sqrt(6) of its largest element.  Both together stay
below 1e-3 of the norm; the rounding of the result is 0.0017, and the framework's bound for such products, 5e-3 of the norm and 2e-2 of the largest element, holds."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block_layer as B
from paper_2410_17043_amd import _lib
from tests import block_checks as K
from tests import harness as H

pytestmark = pytest.mark.gpu
P = H.P
DEV = H.DEV
SILU, GELU, SWIGLU = 0, 1, 2
f32 = np.float32


def to_dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


# ------------------------------------------------------------------------------------------------ rows
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hn", [(1, 128), (3, 256), (5, 1152), (2, 2176), (300, 384), (1, 130944)])
def test_quantised_rows(T, Hn, dtype):
    r = np.random.default_rng([T, Hn])
    v = K.on_grid(r.standard_normal((T, Hn)) * 2.0 ** r.integers(-30, 30, (T, 1)), dtype)
    v[T // 2, :5] = v[T // 2].max() * 2
    rows = torch.full((T, P.moe_int8_row_bytes(Hn)), 0xA5, dtype=torch.uint8, device=DEV)
    P.moe_quantize_int8(to_dev(v.astype(f32)).to(P.TORCH_DTYPE[dtype]), rows)
    assert np.array_equal(rows.cpu().numpy(), B.pack_integer_rows(*B.integer_rows(v)))


def test_rows_that_are_not_finite_or_zero_or_tiny():
    v = np.zeros((6, 256), f32)
    v[0, 3], v[1, 200], v[2, 0] = np.inf, np.nan, -np.inf
    v[3, 5], v[4, 7] = 1e-44, 3.4e38
    rows = torch.empty(6, P.moe_int8_row_bytes(256), dtype=torch.uint8, device=DEV)
    P.moe_quantize_int8(to_dev(v), rows)
    raw = rows.cpu().numpy()
    s = np.ascontiguousarray(raw[:, 256:260]).view(f32)[:, 0]
    assert np.isnan(s[:3]).all() and not raw[:3, :256].any() and not raw[5, :256].any()
    assert s[3] == s[5] == f32(2.0 ** -126) and raw[4, 7] == 127 and not raw[:, 260:].any()


def test_halves_go_to_the_even_number():
    v = np.concatenate([np.arange(-127, 128) / 2.0, [127.0]])[None]
    for dtype in ("bf16", "fp32"):
        rows = torch.empty(1, 384, dtype=torch.uint8, device=DEV)
        P.moe_quantize_int8(to_dev(v.astype(f32)).to(P.TORCH_DTYPE[dtype]), rows)
        assert np.array_equal(rows.cpu().numpy()[0, :256].view(np.int8), np.rint(v[0]))


def test_halves_of_scales_that_are_no_powers_of_two():
    scales = np.concatenate([np.arange(1, 200, 2), 2 ** 16 - np.arange(1, 100, 2)])      # 253 halves of them are 24 bits, their inverses are not exact
    v = np.concatenate([np.arange(-126.5, 127), [127.0, 0.0]])[None] * scales[:, None]
    rows = torch.empty(len(v), 384, dtype=torch.uint8, device=DEV)
    assert np.array_equal(v.astype(f32), v)
    P.moe_quantize_int8(to_dev(v.astype(f32)), rows)
    want = np.broadcast_to(np.rint(v[0]), v.shape)
    assert np.array_equal(rows.cpu().numpy()[:, :256].view(np.int8), want)


# ------------------------------------------------------------------------------------------------ FFN
def make_experts(r, n, Hn, F, act, positive=True):
    lo = 0 if positive else -127
    out = []
    for _ in range(n):
        e = {"w1": r.integers(lo, 128, (F, Hn)).astype(np.int8), "w_up": None, "s_up": None, "w_down": r.integers(-127, 128, (Hn, F)).astype(np.int8)}
        scale = 1.0 if positive else 0.02 / 127
        e["s1"] = (r.uniform(0.5, 2.0, F) * scale).astype(f32)
        e["s_down"] = (r.uniform(0.5, 2.0, Hn) * 0.02 / 127).astype(f32)
        if act == SWIGLU:
            e["w_up"], e["s_up"] = r.integers(-127, 128, (F, Hn)).astype(np.int8), (r.uniform(0.5, 2.0, F) * 0.02 / 127).astype(f32)
        out.append(e)
    return out


def make_rows(r, R, Hn, positive=True):
    q = r.integers(0 if positive else -127, 128, (R, Hn)).astype(np.int8)
    return q, (r.uniform(0.5, 2.0, R) * (1.0 if positive else 1.0 / 60)).astype(f32)


def bits_of(q, s, e, act):
    """What the FFN has to give for arguments of an activation that are zero or large, as bf16 numbers."""
    product = lambda x, w: (x.astype(np.float64) @ w.astype(np.float64).T).astype(f32)  # noqa: E731
    a = product(q, e["w1"]) * e["s1"] * s[:, None]
    assert np.all((a == 0) | (a > 40)) and np.all(a < 1e30)
    h = a * (product(q, e["w_up"]) * e["s_up"] * s[:, None]) if act == SWIGLU else a
    hq, hs = B.integer_rows(B.round_bf16(h))
    return B.round_bf16(product(hq, e["w_down"]) * e["s_down"] * hs[:, None])



def on_device(experts):
    return [{k: None if v is None else to_dev(v) for k, v in e.items()} for e in experts]


def run_ffn(rows, so, se, d_experts, Hn, F, act):
    R = rows.shape[0]
    out = torch.full((R, Hn), -7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((P.moe_ffn_int8_workspace_bytes(R, Hn, F, act),), 0xFF, dtype=torch.uint8, device=DEV)
    P.moe_expert_ffn_int8(rows, R, to_dev(np.asarray(so, np.int32)), to_dev(np.asarray(se, np.int32)), len(se), d_experts, Hn, F, act, out, ws)
    torch.cuda.synchronize()
    return out


def check_bits(r, R, Hn, F, act, so, se, n_local):
    q, s = make_rows(r, R, Hn)
    if R > 2:
        q[R // 2] = 0
    experts = make_experts(r, n_local, Hn, F, act)
    out = run_ffn(to_dev(B.pack_integer_rows(q, s)), so, se, on_device(experts), Hn, F, act).double().cpu().numpy()
    want = np.full((R, Hn), -7.0)                                            # rows outside every segment stay as they were
    for i, e in enumerate(se):
        a, b = so[i], so[i + 1]
        if 0 <= e < n_local and b > a:
            want[a:b] = bits_of(q[a:b], s[a:b], experts[e], act)
    assert np.array_equal(out, want)


@pytest.mark.parametrize("act", [SILU, GELU, SWIGLU])
@pytest.mark.parametrize("R,Hn,F", [(1, 128, 128), (2, 256, 128), (17, 128, 384), (33, 384, 640), (64, 256, 256), (65, 1152, 256), (129, 256, 1408), (300, 640, 512)])
def test_one_expert(R, Hn, F, act):
    check_bits(np.random.default_rng([R, Hn, F, act]), R, Hn, F, act, [0, R], [0], 1)


@pytest.mark.parametrize("seg_rows,seg_expert,n_local", [
    ([0, 5, 0, 1], [0, 1, 2, 1], 3),                                         # empty segments
    ([3] * 24, [i % 4 for i in range(24)], 4),                               # gathered rows of many short segments
    ([40, 90, 1, 70, 33], [2, 0, 2, 0, 1], 4),                               # an expert without rows
    ([7, 9, 11], [0, 9, -1], 2),                                             # experts that do not exist
    ([2] * 130, [(i * 5) % 7 for i in range(130)], 7),                       # more than 64 segments
    ([257, 300], [1, 0], 2),
    ([2] * 699 + [13], [i % 4 for i in range(700)], 4)])                     # tile maps of two heights do not fit beside each other
def test_segments(seg_rows, seg_expert, n_local):
    r = np.random.default_rng(len(seg_rows))
    so = np.concatenate([[3], 3 + np.cumsum(seg_rows)])                      # three rows in front and two behind belong to no segment
    check_bits(r, int(so[-1]) + 2, 256, 384, SWIGLU, so, seg_expert, n_local)


def plan_of(R, n_used, nseg, Hn, F, act):
    p = (C.c_int32 * 5)()
    assert _lib.load().moe_selfcheck_fp8_plan(R, n_used, nseg, Hn, F, act, 256, p) == 0
    return dict(zip(("mt", "bm1", "bm2", "deep", "pieces"), p))


@pytest.mark.parametrize("R,Hn,F,act,n_local,want", [
    (5, 1024, 8192, SWIGLU, 1, dict(mt=1)), (20, 1024, 8192, GELU, 1, dict(mt=2)), (60, 896, 8064, SWIGLU, 1, dict(mt=4)),
    (9, 256, 4096, GELU, 1, dict(mt=1)), (20, 896, 8064, SWIGLU, 1, dict(mt=2)), (9, 896, 8064, SILU, 1, dict(mt=1)), (60, 896, 8064, GELU, 1, dict(mt=4)),
    (100, 256, 4096, SILU, 2, dict(mt=4, pieces=8)),
    (1100, 128, 14336, GELU, 1, dict(mt=0, bm2=256, pieces=7)), (1300, 384, 8192, SWIGLU, 2, dict(mt=0, bm2=256, pieces=8)),
    (1200, 512, 640, SWIGLU, 3, dict(mt=0, bm1=64, bm2=128, deep=1)), (9000, 384, 1408, SWIGLU, 2, dict(mt=0, bm1=256)),
    (9000, 256, 2304, SILU, 2, dict(mt=0, bm1=128)), (3000, 512, 1408, SWIGLU, 1, dict(mt=0, bm2=128))])
def test_every_kernel(R, Hn, F, act, n_local, want):
    plan = plan_of(R, n_local, n_local, Hn, F, act)
    assert {k: plan[k] for k in want} == want, plan
    check_bits(np.random.default_rng([R, F]), R, Hn, F, act, [R * i // n_local for i in range(n_local + 1)], list(range(n_local)), n_local)


@pytest.mark.parametrize("Hn,F,n_local,nseg,most,act", [
    (2048, 1408, 1, 3, 5, SWIGLU),                                           # a map of tiles, the first GEMM cut along K
    (256, 1408, 8, 64, 2, SWIGLU), (1152, 1408, 8, 20, 5, SILU),             # the list itself, 64 columns a block
    (256, 1408, 16, 64, 4, GELU), (1152, 1408, 24, 33, 6, SWIGLU),           # 128 columns a block
    (256, 1408, 8, 65, 2, SILU), (256, 1408, 16, 70, 2, SWIGLU),             # more than 64 segments: a map, either width
    (256, 1408, 24, 130, 3, SWIGLU),                                         # tiles that do not stream
    (640, 14336, 1, 64, 2, SWIGLU)])                                         # one expert, its tiles put together from many segments
def test_few_rows_in_many_segments(Hn, F, n_local, nseg, most, act):
    r = np.random.default_rng([Hn, F, nseg])
    seg_rows = r.integers(0, most + 1, nseg)
    so = np.concatenate([[2], 2 + np.cumsum(seg_rows)])
    R = int(so[-1]) + 1
    assert (plan_of(R, min(n_local, nseg), nseg, Hn, F, act)["mt"] > 0) == (nseg < 130)
    check_bits(r, R, Hn, F, act, so, r.integers(-1, n_local + 1, nseg), n_local)
    check_bits(r, R, Hn, F, act, np.full(nseg + 1, R // 2), np.zeros(nseg, int), n_local)   # nothing arrived


@pytest.mark.parametrize("R,Hn,F,act,n_local,nseg", [(403, 2048, 1408, SWIGLU, 4, 64), (37, 1024, 2304, SWIGLU, 1, 8), (700, 1152, 2304, SILU, 4, 24), (1500, 1024, 1024, GELU, 3, 12),
                                                     (90, 2048, 1408, SWIGLU, 8, 16), (2200, 512, 640, SWIGLU, 2, 4)])
def test_ordinary_weights(R, Hn, F, act, n_local, nseg):
    r = np.random.default_rng(R)
    so = np.concatenate([[0], np.sort(r.integers(0, R + 1, nseg - 1)), [R]])
    se = r.integers(0, n_local, nseg)
    q, s = make_rows(r, R, Hn, False)
    experts = make_experts(r, n_local, Hn, F, act, False)
    out = run_ffn(to_dev(B.pack_integer_rows(q, s)), so, se, on_device(experts), Hn, F, act).double().cpu().numpy()
    want = np.concatenate([B.expert_ffn_int8(q[a:b], s[a:b], experts[e], act) for a, b, e in zip(so[:-1], so[1:], se)])
    H.assert_close(out, want, "bf16")


def test_rows_that_stand_for_nan_stay_by_themselves():
    r = np.random.default_rng(4)
    q, s = make_rows(r, 90, 256)
    d = on_device(make_experts(r, 2, 256, 384, SWIGLU))
    clean = run_ffn(to_dev(B.pack_integer_rows(q, s)), [0, 40, 90], [1, 0], d, 256, 384, SWIGLU)
    s[[3, 50]] = np.nan
    got = run_ffn(to_dev(B.pack_integer_rows(q, s)), [0, 40, 90], [1, 0], d, 256, 384, SWIGLU)
    keep = [i for i in range(90) if i not in (3, 50)]
    assert got[[3, 50]].isnan().all() and torch.equal(got[keep], clean[keep])


def test_a_row_does_not_depend_on_the_others():
    # alone (streamed), among a hundred (streamed in taller tiles, cut along K), among thousands (tiles)
    r = np.random.default_rng(5)
    Hn, F = 512, 4096
    q, s = make_rows(r, 5000, Hn, False)
    rows, d = to_dev(B.pack_integer_rows(q, s)), on_device(make_experts(r, 1, Hn, F, SWIGLU, False))
    whole = run_ffn(rows, [0, 5000], [0], d, Hn, F, SWIGLU)
    for n in (1, 7, 20, 100, 700, 1500):
        assert torch.equal(run_ffn(rows[:n].contiguous(), [0, n], [0], d, Hn, F, SWIGLU), whole[:n])


def test_largest_sums():
    # 127 * 127 * K and the lowest value on both sides: whole numbers up to 2^31
    Hn, F, R = 130944, 128, 3
    q = np.full((R, Hn), 127, np.int8)
    q[1], q[2, ::2] = -127, -127
    e = {"w1": np.full((F, Hn), 127, np.int8), "w_up": None, "s_up": None, "s1": np.full(F, 1e-6, f32), "w_down": np.ones((Hn, F), np.int8), "s_down": np.ones(Hn, f32)}
    e["w1"][1] = -128
    out = run_ffn(to_dev(B.pack_integer_rows(q, np.ones(R, f32))), [0, R], [0], on_device([e]), Hn, F, SILU).double().cpu().numpy()
    H.assert_close(out, B.expert_ffn_int8(q, np.ones(R, f32), e, SILU), "bf16")


def test_replayed_in_a_graph_on_another_stream():
    r = np.random.default_rng(14)
    Hn, F, R = 1024, 768, 500
    experts = on_device(make_experts(r, 3, Hn, F, SWIGLU, False))
    so, se = to_dev(np.array([0, 100, 333, 400, R], np.int32)), to_dev(np.array([0, 2, 0, 1], np.int32))
    recv = to_dev(B.pack_integer_rows(*make_rows(r, R, Hn, False)))
    ws = torch.full((P.moe_ffn_int8_workspace_bytes(R, Hn, F, SWIGLU),), 0xFF, dtype=torch.uint8, device=DEV)
    outs = [torch.full((R, Hn), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        call = P.bind_expert_ffn_int8(recv, R, so, se, 4, experts, Hn, F, SWIGLU, outs[1], ws)
        call()
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            call(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        recv.copy_(to_dev(B.pack_integer_rows(*make_rows(r, R, Hn, False))))
        outs[1].fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        P.moe_expert_ffn_int8(recv, R, so, se, 4, experts, Hn, F, SWIGLU, outs[0], ws)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and not torch.isnan(outs[0]).any()


def test_arrays_beyond_4_gib():
    n, R, Hn, F, act = 8192, 560000, 7680, 128, SILU
    assert R * P.moe_int8_row_bytes(Hn) > 2 ** 32                            # rows are no longer gathered: tiles of adjacent rows only
    r = np.random.default_rng(32)
    q, s = make_rows(r, n, Hn)
    experts = make_experts(r, 2, Hn, F, act)
    recv = to_dev(B.pack_integer_rows(q, s)).repeat(-(-R // n), 1)[:R]
    out = run_ffn(recv, [0, 200001, 400003, R], [1, 0, 1], on_device(experts), Hn, F, act)
    pitch = P.moe_int8_row_bytes(Hn)
    for owner, some in ((1, [0, 1, n - 1, 200000, 400003, 2 ** 32 // pitch, 2 ** 32 // pitch + 1, R - 1]), (0, [200001, 2 ** 32 // (2 * Hn), 2 ** 32 // (2 * Hn) + 1, 400002])):
        at = [i % n for i in some]
        assert np.array_equal(out[some].double().cpu().numpy(), bits_of(q[at], s[at], experts[owner], act))


def test_a_share_in_integers_from_the_residual_stream_to_the_next():
    """norm of a block -> gate -> dispatch of the packed rows -> experts -> combine and the next norms, as a layer between two others runs them."""
    r = np.random.default_rng(7)
    T, Hn, F, E, k = 70, 384, 256, 8, 2
    bf = lambda *n: to_dev(K.on_grid(r.standard_normal(n), "bf16").astype(f32)).bfloat16()  # noqa: E731
    y, residual, w_gate = bf(T, Hn), bf(T, Hn), bf(E, Hn) * 0.05
    gamma = bf(Hn)
    experts = make_experts(r, E, Hn, F, SWIGLU, False)
    r1, normed = torch.empty_like(y), torch.empty_like(y)
    rows = torch.empty(T, P.moe_int8_row_bytes(Hn), dtype=torch.uint8, device=DEV)
    before = P.block_rule(scale=0.5, gamma_pre=gamma)
    P.moe_block_norm(y, residual, before, r1, normed, rows, P.ROWS_INT8)
    i32 = lambda *n: torch.empty(*n, dtype=torch.int32, device=DEV)  # noqa: E731
    idx, w = i32(T, k), torch.empty(T, k, device=DEV)
    gate, wire = P.MoeCtx(T, Hn, E, k, 1, "bf16", 1), P.MoeCtx(T, rows.shape[1] // 2, E, k, 1, "bf16", 1)
    P.moe_route(gate, normed, w_gate, None, idx, w)
    S = T * k
    send, s2r, r2s, so, se = torch.empty(S, rows.shape[1], dtype=torch.uint8, device=DEV), i32(S), i32(S), i32(E + 1), i32(E)
    P.moe_dispatch(wire, rows.view(torch.bfloat16), idx, [0] * E, [0], send.view(torch.bfloat16), s2r, r2s, so, se)
    out, ws = torch.empty(S, Hn, dtype=torch.bfloat16, device=DEV), torch.empty(P.moe_ffn_int8_workspace_bytes(S, Hn, F, SWIGLU), dtype=torch.uint8, device=DEV)
    P.moe_expert_ffn_int8(send, S, so, se, E, on_device(experts), Hn, F, SWIGLU, out, ws)
    r2, rows2 = torch.empty_like(y), torch.empty_like(rows)
    P.moe_combine_norm(gate, out, s2r, w, None, r1, P.block_rule(gamma_pre=gamma), r2, None, rows2, P.ROWS_INT8)
    raw = rows.cpu().numpy()
    q, s = raw[:, :Hn].view(np.int8), np.ascontiguousarray(raw[:, Hn:Hn + 4]).view(f32)[:, 0]
    K.assert_integer_rows(raw, B.normed(r1.double().cpu().numpy(), gamma.double().cpu().numpy(), 1e-6))
    layer = np.zeros((T, Hn))
    for t in range(T):
        for j in range(k):
            layer[t] += w[t, j].item() * B.expert_ffn_int8(q[t:t + 1], s[t:t + 1], experts[idx[t, j].item()], SWIGLU)[0]
    want = B.residual_sum(layer, r1.double().cpu().numpy(), None, None, 0, 1.0, True, 1e-6)
    H.assert_close(r2.double().cpu().numpy(), want, "bf16")
    K.assert_integer_rows(rows2.cpu().numpy(), B.normed(r2.double().cpu().numpy(), gamma.double().cpu().numpy(), 1e-6))
