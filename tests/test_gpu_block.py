"""The norms behind and in front of a block, with gate and residual scale, on the GPU against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import block_layer as B
from tests import block_checks as K
from tests import harness as H

pytestmark = pytest.mark.gpu
P = H.P
DEV = H.DEV
EPS = 1e-6


def dev(v, dtype):
    return None if v is None else torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(DEV).to(P.TORCH_DTYPE[dtype])


def host(t):
    return t.double().cpu().numpy()


class Case:
    """Inputs of one call (float64 on the grid of their type) and what it has to give."""

    def __init__(self, T, Hn, dtype, post=True, gate_tokens=0, scale=1.0, residual=True, gammas=True, k=0, shared=False, dropped=0.1, seed=0, eps=EPS):
        rng = np.random.default_rng([T, Hn, k, seed])
        g = lambda *s: K.on_grid(rng.standard_normal(s), dtype)  # noqa: E731
        self.T, self.H, self.dtype, self.post, self.scale, self.k, self.eps = T, Hn, dtype, post, scale, k, eps
        self.residual = g(T, Hn) * 4.0 if residual else None
        self.gamma_post = 1.0 + 0.25 * K.on_grid(rng.integers(-2, 3, Hn), dtype) if gammas and post else None
        self.gamma_pre = K.on_grid(1.0 + 0.1 * rng.standard_normal(Hn), dtype) if gammas else None
        self.gate_tokens = gate_tokens
        self.gate = g(-(-T // gate_tokens), Hn) if gate_tokens else None
        if k:
            self.ret = g(T * k, Hn)
            rows = rng.permutation(T * k).astype(np.int32)
            rows[rng.random(T * k) < dropped] = -1
            self.slot_to_row = rows.reshape(T, k)
            self.topk_w = rng.random((T, k)).astype(np.float32)
            self.shared = g(T, Hn) if shared else None
        else:
            self.y = g(T, Hn)

    def output(self):
        return B.combine(self.ret, self.slot_to_row, self.topk_w, self.shared) if self.k else self.y

    def rule(self):
        return P.block_rule(self.post, dev(self.gamma_post, self.dtype), dev(self.gate, self.dtype), self.gate_tokens, self.scale, dev(self.gamma_pre, self.dtype), self.eps)

    def call(self, residual_out, normed, rows, form=P.ROWS_FP8, rule=None):
        rule = rule or self.rule()
        if self.k:
            ctx = P.MoeCtx(self.T, self.H, max(self.k, 8), self.k, 1, self.dtype)
            bound = P.bind_combine_norm(ctx, dev(self.ret, self.dtype), torch.from_numpy(self.slot_to_row).to(DEV), torch.from_numpy(self.topk_w).to(DEV),
                                        dev(self.shared, self.dtype), dev(self.residual, self.dtype), rule, residual_out, normed, rows, form)
        else:
            bound = P.bind_block_norm(dev(self.y, self.dtype), dev(self.residual, self.dtype), rule, residual_out, normed, rows, form)
        return bound

    def buffers(self, form):
        e = lambda: torch.full((self.T, self.H), 7.0, device=DEV, dtype=P.TORCH_DTYPE[self.dtype])  # noqa: E731
        pitch = {None: 0, P.ROWS_INT8: P.moe_int8_row_bytes(self.H), P.ROWS_FP8: P.moe_fp8_row_bytes(self.H)}[form]
        return e(), e(), torch.full((self.T, pitch), 0xA5, device=DEV, dtype=torch.uint8) if pitch else None

    def check(self, form=None):
        r, v, rows = self.buffers(form)
        self.call(r, v, rows, form or 0)()
        torch.cuda.synchronize()
        self.check_results(r, v, rows, form)

    def check_results(self, r, v, rows, form):
        want = B.residual_sum(self.output(), self.residual, self.gamma_post, self.gate, self.gate_tokens, self.scale, self.post, self.eps)
        K.assert_rounded(host(r), want, self.dtype)
        want = B.normed(host(r), self.gamma_pre, self.eps)
        if v is not None:
            K.assert_rounded(host(v), want, self.dtype)
        if rows is not None:
            (K.assert_integer_rows if form == P.ROWS_INT8 else K.assert_e4m3_rows)(rows.cpu().numpy(), want)


# one lane's elements, parts of a chunk, several chunks and waves, two and four chunks a wave
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hn", [(1, 8), (3, 24), (5, 520), (9, 1032), (257, 1152), (2, 8184), (3, 8712), (2, 16400), (1, 32768)])
def test_block_norm_sizes(dtype, T, Hn):
    Case(T, Hn, dtype, gate_tokens=2, scale=0.22).check()


@pytest.mark.parametrize("Hn", [4, 12, 508, 1028, 2052])
def test_fp32_rows_that_end_inside_a_lane(Hn):
    Case(5, Hn, "fp32", gate_tokens=5).check()
    Case(3, Hn, "fp32", k=3, shared=True).check()


@pytest.mark.parametrize("form", [None, P.ROWS_FP8, P.ROWS_INT8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,Hn", [(1, 128), (6, 384), (7, 640), (33, 2176), (3, 8320), (2, 17024)])
def test_rows_of_both_formats(form, dtype, T, Hn):
    Case(T, Hn, dtype, seed=1).check(form)
    Case(T, Hn, dtype, k=2, shared=True, seed=2).check(form)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("post,gate_tokens,scale,residual,gammas", [(True, 0, 1.0, True, False), (False, 0, -0.5, True, True), (False, 1, 2.0, False, False), (True, 3, 1.0, False, True),
                                                                   (True, 50, 0.0, True, True), (False, 50, 1.0, True, False)])
def test_parts_of_the_rule(dtype, post, gate_tokens, scale, residual, gammas):
    Case(50, 768, dtype, post, gate_tokens, scale, residual, gammas).check(P.ROWS_INT8)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("k", [1, 2, 3, 4, 5, 6, 8, 16])
def test_combined_rows(dtype, k):
    Case(19, 640, dtype, k=k, shared=k % 2 == 0, gate_tokens=19).check()
    Case(5, 256, dtype, k=k, dropped=1.1, shared=k % 2 == 1).check(P.ROWS_INT8)          # no slot is kept


def test_dropped_slots_do_not_touch_rows():
    # slots that are dropped, and row 0, which nobody chose, hold NaN
    c = Case(8, 256, "bf16", k=2)
    c.slot_to_row[:] = np.arange(16).reshape(8, 2)
    c.slot_to_row[0, 0] = c.slot_to_row[3] = -1
    c.ret[0] = np.nan
    c.check(P.ROWS_INT8)


@pytest.mark.parametrize("form", [P.ROWS_FP8, P.ROWS_INT8])
def test_infinities_and_nan_stay_in_their_rows(form):
    c = Case(8, 512, "bf16", gammas=False)
    c.y[1, 5] = np.inf
    c.y[2, 7] = np.nan
    c.residual[4, 500] = -np.inf
    c.y[5], c.residual[5] = 0.0, 0.0
    r, v, rows = c.buffers(form)
    c.call(r, v, rows, form)()
    torch.cuda.synchronize()
    r, v = host(r), host(v)
    # an infinite sum: finite elements become zeros, infinite ones NaN
    assert np.isnan(r[1, 5]) and np.array_equal(np.delete(r[1], 5), np.delete(c.residual[1], 5)) and np.isnan(v[1]).all()
    assert np.isnan(r[2]).all() and np.isnan(v[2]).all()
    assert r[4, 500] == -np.inf and np.isnan(v[4, 500]) and not np.delete(v[4], 500).any()
    assert not v[5].any()
    raw = rows.cpu().numpy()
    if form == P.ROWS_INT8:
        s = np.ascontiguousarray(raw[:, 512:516]).view(np.float32)[:, 0]
        assert np.array_equal(np.isnan(s), [False, True, True, False, True, False, False, False]) and s[5] == np.float32(2.0 ** -126)
        assert not raw[[1, 2, 4, 5], :512].any()
    fine = [0, 3, 6, 7]
    K.assert_rounded(v[fine], B.normed(r[fine], None, c.eps), "bf16")
    (K.assert_integer_rows if form == P.ROWS_INT8 else K.assert_e4m3_rows)(raw[fine], B.normed(r[fine], None, c.eps))


def test_extreme_values():
    # sums of squares beyond and below fp32, eps zero
    for factor, eps in ((1e36, 0.0), (1e-30, 0.0), (1e-30, 1e-6)):
        c = Case(6, 384, "fp32", scale=1.0, eps=eps)
        c.y, c.residual = K.on_grid(c.y * factor, "fp32"), K.on_grid(c.residual * factor, "fp32")
        c.check(P.ROWS_INT8)
        c.check(P.ROWS_FP8)


def test_integer_rows_at_the_middle_of_two_numbers():
    # the norm gives one, so v is gamma: halves go to the even number
    Hn = 256
    c = Case(1, Hn, "fp32", post=False, gammas=False, eps=0.0)
    c.y, c.residual = np.ones((1, Hn)), np.zeros((1, Hn))
    c.gamma_pre = np.concatenate([np.arange(-127, 128) / 2.0, [127.0]])
    r, v, rows = c.buffers(P.ROWS_INT8)
    c.call(r, v, rows, P.ROWS_INT8)()
    assert np.array_equal(rows.cpu().numpy()[0, :Hn].view(np.int8), np.rint(c.gamma_pre)) and rows[0, Hn:Hn + 4].view(torch.float32).item() == 1.0


@pytest.mark.parametrize("which", ["y", "residual", "both"])
def test_results_in_place(which):
    c = Case(37, 1152, "bf16", gate_tokens=10, scale=0.5)
    y, res = dev(c.y, "bf16"), dev(c.residual, "bf16")
    out, normed = {"y": (y, torch.empty_like(y)), "residual": (res, torch.empty_like(y)), "both": (res, y)}[which]
    P.moe_block_norm(y, res, c.rule(), out, normed, None)
    c.check_results(out, normed, None, None)


def test_one_output_alone():
    c = Case(9, 640, "bf16", k=2)
    r, v, rows = c.buffers(P.ROWS_INT8)
    c.call(r, v, rows, P.ROWS_INT8)()
    for keep in range(3):
        some = [t if i == keep else None for i, t in enumerate(c.buffers(P.ROWS_INT8))]
        c.call(*some, P.ROWS_INT8)()
        assert torch.equal(some[keep], (r, v, rows)[keep])


def test_no_tokens():
    e = torch.empty(0, 256, device=DEV, dtype=torch.bfloat16)
    P.moe_block_norm(e, None, P.block_rule(), e.clone(), None, None)


def test_arrays_beyond_4_gib():
    T, Hn = 70000, 32768
    y = torch.zeros(T, Hn, device=DEV, dtype=torch.bfloat16)
    rng = np.random.default_rng(5)
    some = [0, 32767, 32768, 65535, 65536, T - 1]
    values = K.on_grid(rng.standard_normal((len(some), Hn)), "bf16")
    y[some] = dev(values, "bf16")
    gate = K.on_grid(rng.standard_normal((2, Hn)), "bf16")
    rows = torch.empty(T, P.moe_int8_row_bytes(Hn), dtype=torch.uint8, device=DEV)
    P.moe_block_norm(y, None, P.block_rule(True, None, dev(gate, "bf16"), 65536, 1.0, None, EPS), y, None, rows, P.ROWS_INT8)
    r = host(y[some])
    K.assert_rounded(r, B.residual_sum(values, None, None, gate[[0, 0, 0, 0, 1, 1]], 1, 1.0, True, EPS), "bf16")
    K.assert_integer_rows(rows[some].cpu().numpy(), B.normed(r, None, EPS))
    assert not rows[1, :Hn].any()


def test_captured_and_replayed_on_another_stream():
    c = Case(64, 2048, "bf16", k=6, shared=True, gate_tokens=64)
    eager = c.buffers(P.ROWS_FP8)
    c.call(*eager, P.ROWS_FP8)()
    torch.cuda.synchronize()
    r, v, rows = c.buffers(P.ROWS_FP8)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call = c.call(r, v, rows, P.ROWS_FP8)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        for t in (r, v, rows):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((r, v, rows), eager))


def test_same_result_in_every_place():
    # a token's result does not hang on its row or the number of tokens
    c = Case(4, 1536, "bf16", k=3)
    r, v, rows = c.buffers(P.ROWS_INT8)
    c.call(r, v, rows, P.ROWS_INT8)()
    for t in range(4):
        one = Case(1, 1536, "bf16", k=3)
        one.ret, one.slot_to_row, one.topk_w = c.ret, c.slot_to_row[t:t + 1], c.topk_w[t:t + 1]
        one.residual, one.gamma_post, one.gamma_pre, one.shared = c.residual[t:t + 1], c.gamma_post, c.gamma_pre, None
        got = one.buffers(P.ROWS_INT8)
        one.call(*got, P.ROWS_INT8)()
        assert all(torch.equal(a[0], b[t]) for a, b in zip(got, (r, v, rows)))
