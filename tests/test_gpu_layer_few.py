"""The whole layer for a few tokens on the GPU against the oracle in 64 bits.

Tolerances.  Choices have to be the oracle's where its margins exceed 1e-9 (logits are 64-bit sums).  Weights: exponentials and quotients in 64 bits, rounded once: 2^-24 of
the value, and 1e-12.  y: bf16 rounds the result (2^-8 of each element, by independent amounts: 2^-8 / sqrt(3) of their norm, about 0.0023, on a logarithmic scale somewhat less: 0.0017); the inner
activations are kept to 2^-17, and fp32 sums add little.  The framework's bound for products that round those too, 5e-3 of the norm and 2e-2 of the largest element
(tests/harness.py), holds; what is rounded is looked at in tests/test_gpu_layer_few_rounding.py.  fp32: 1e-6 and 1e-5, the same."""
import numpy as np
import pytest
import torch

from oracle import block_layer as B
from oracle import moe_layer as O
from tests import harness as H
from tests.block_checks import assert_rounded, on_grid

pytestmark = pytest.mark.gpu
P = H.P
DEV = H.DEV


def dev(v, dtype):
    return None if v is None else torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(DEV).to(P.TORCH_DTYPE[dtype])


class Layer:
    def __init__(self, T, Hn, F, E, k, dtype="bf16", act=2, local=None, F_shared=0, renorm=0, bias=True, seed=0):
        rng = np.random.default_rng([T, Hn, F, E, k, seed])
        g = lambda s, *n: on_grid(s * rng.standard_normal(n), dtype)  # noqa: E731
        self.T, self.H, self.F, self.E, self.k, self.dtype, self.act, self.F_shared, self.renorm = T, Hn, F, E, k, dtype, act, F_shared, renorm
        self.local = list(range(E)) if local is None else local
        n = max(self.local + [-1]) + 1
        scale = 1.0 / np.sqrt(Hn)
        weights = lambda f: {"w1": g(scale, f, Hn), "w_up": g(scale, f, Hn) if act == 2 else None, "w_down": g(1.0 / np.sqrt(f), Hn, f)}  # noqa: E731
        self.experts = [weights(F) for _ in range(n)]
        self.shared = weights(F_shared) if F_shared else None
        self.x, self.w_gate = g(1.0, T, Hn), g(scale, E, Hn)
        self.bias = rng.standard_normal(E).astype(np.float32) if bias else None
        self.ctx = P.MoeCtx(T, Hn, E, k, 1, dtype, renorm)

    def device(self):
        d = lambda w: {n: dev(v, self.dtype) for n, v in w.items()}  # noqa: E731
        self.d_experts, self.d_shared = [d(w) for w in self.experts], d(self.shared) if self.shared else None
        self.d_x, self.d_gate = dev(self.x, self.dtype), dev(self.w_gate, self.dtype)
        self.d_bias = None if self.bias is None else torch.from_numpy(self.bias).to(DEV)
        self.ws = torch.full((P.moe_layer_few_workspace_bytes(self.ctx, self.F, self.F_shared),), 0xFF, dtype=torch.uint8, device=DEV)
        self.idx = torch.full((self.T, self.k), -7, dtype=torch.int32, device=DEV)
        self.w = torch.full((self.T, self.k), np.nan, dtype=torch.float32, device=DEV)
        self.y = torch.full((self.T, self.H), np.nan, dtype=P.TORCH_DTYPE[self.dtype], device=DEV)
        return self

    def bind(self, routed=False):
        return P.bind_layer_few(self.ctx, self.d_x, None if routed else self.d_gate, None if routed else self.d_bias, self.idx, self.w, self.d_experts, self.local, self.F,
                                self.act, self.d_shared, self.F_shared, self.y, self.ws)

    def want(self, idx, w):
        return B.layer_few(self.x, idx, w, self.experts, self.local, self.act, self.shared)

    def check(self, gate=True):
        """Runs the layer, or (without gate) looks at what has run."""
        if gate:
            self.device().bind()()
            idx, w, z = O.route(self.x, self.w_gate, self.bias, self.k, self.renorm)
            assert O.route_margin(z, self.k).min() > 1e-9
            assert np.array_equal(self.idx.cpu().numpy(), idx)
            got = self.w.double().cpu().numpy()
            assert np.all(np.abs(got - w) <= (2.0 ** -24 + 1e-12) * w + 1e-45)
        H.assert_close(H.host(self.y), self.want(self.idx.cpu().numpy(), self.w.cpu().numpy()), self.dtype)
        return self


@pytest.mark.parametrize("T", [1, 2, 3, 5, 15, 16, 17, 31, 33, 48, 64])
@pytest.mark.parametrize("act", [0, 1, 2])
def test_tokens_and_activations(T, act):
    Layer(T, 256, 384, 8, 2, act=act, F_shared=128 if T % 2 else 0, renorm=T % 2).check()


@pytest.mark.parametrize("T,Hn,F,E,k", [(1, 128, 128, 1, 1), (1, 2048, 1408, 64, 6), (4, 1152, 2304, 24, 3), (64, 640, 256, 64, 16), (7, 128, 1152, 5, 5), (9, 4096, 256, 8, 2), (3, 512, 4096, 3, 1)])
def test_sizes(T, Hn, F, E, k):
    Layer(T, Hn, F, E, k).check()


# widths that end inside 128 bytes, inside 16 rows
@pytest.mark.parametrize("T,Hn,F,Fs", [(1, 4, 4, 0), (1, 64, 128, 0), (2, 36, 20, 4), (20, 100, 132, 12), (64, 260, 68, 0), (5, 1028, 516, 260), (33, 32, 1000, 28)])
def test_fp32_widths(T, Hn, F, Fs):
    for act in range(3):
        Layer(T, Hn, F, 6, 2, "fp32", act, F_shared=Fs, renorm=1).check()


@pytest.mark.parametrize("E", [1, 2, 63, 64, 65, 200, 256])
@pytest.mark.parametrize("T", [1, 6])
def test_experts_of_the_gate(E, T):
    local = [e % 3 if e < 3 else -1 for e in range(E)]
    Layer(T, 128, 128, E, min(E, 8), local=local, bias=E % 2 == 0).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_experts_on_other_gpus(dtype):
    # places in any order; the parts of two GPUs add up to the layer (64 bits: the sum of the oracle's parts is the whole)
    here = [-1, 2, -1, 0, 1, -1, 3, -1]
    Layer(17, 256, 128, 8, 3, dtype, local=here, F_shared=256).check()
    # nothing chosen is here: zeros, or the shared expert alone
    for Fs in (0, 128):
        c = Layer(5, 256, 128, 8, 2, dtype, local=[0] + [-1] * 7, F_shared=Fs)
        c.bias = np.array([-1e9] + [0.0] * 7, np.float32)
        c.check()
    c = Layer(5, 256, 128, 8, 2, dtype, local=[-1] * 8)
    c.check()
    assert not c.y.any()
    Layer(5, 256, 128, 8, 2, dtype, local=[-1] * 8, F_shared=128).check()


def test_given_choices():
    c = Layer(19, 256, 384, 8, 4, F_shared=128).device()
    rng = np.random.default_rng(3)
    idx = rng.integers(-2, 10, (19, 4)).astype(np.int32)                     # outside [0, 8): nobody
    idx[4] = -1
    idx[5] = 3                                                               # one expert four times
    idx[6, 1:3] = idx[6, 0] = 2
    c.idx.copy_(torch.from_numpy(idx))
    c.w.copy_(torch.from_numpy(rng.random((19, 4)).astype(np.float32)))
    c.bind(routed=True)()
    c.check(gate=False)
    assert np.array_equal(c.idx.cpu().numpy(), idx)


def test_equal_logits_go_to_the_lower_expert():
    c = Layer(5, 128, 128, 70, 6, bias=False, local=[0] + [-1] * 69)
    c.w_gate[:] = c.w_gate[0]
    c.device().bind()()
    assert np.array_equal(c.idx.cpu().numpy(), np.tile(np.arange(6, dtype=np.int32), (5, 1)))
    assert torch.equal(c.w, torch.full((5, 6), 1.0 / 70.0, device=DEV))
    c = Layer(4, 128, 128, 8, 8)                                             # experts out of service come last
    c.bias = np.array([0.0, -np.inf, 0.0, 0.0, -np.inf, 0.0, 0.0, 0.0], np.float32)
    c.device().bind()()
    assert np.array_equal(c.idx[:, 6:].cpu().numpy(), [[1, 4]] * 4) and not c.w[:, 6:].any()


def test_nan_stays_in_its_token():
    c = Layer(6, 256, 256, 8, 2).device()
    c.bind()()
    before, idx = c.y.clone(), c.idx.clone()
    c.d_x[2, 3] = np.nan
    c.bind()()
    assert c.y[2].isnan().all() and ((c.idx[2] >= 0) & (c.idx[2] < 8)).all() and c.idx[2, 0] != c.idx[2, 1]
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(c.y[keep], before[keep]) and torch.equal(c.idx[keep], idx[keep])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_token_does_not_depend_on_the_others(dtype):
    c = Layer(64, 384, 256, 8, 2, dtype, F_shared=128).device()
    c.bind()()
    for n in (1, 2, 16, 17, 32):
        d = Layer(n, 384, 256, 8, 2, dtype, F_shared=128)
        d.x, d.w_gate, d.bias, d.experts, d.shared = c.x[64 - n:], c.w_gate, c.bias, c.experts, c.shared
        d.device().bind()()
        assert torch.equal(d.y, c.y[64 - n:]) and torch.equal(d.idx, c.idx[64 - n:]) and torch.equal(d.w, c.w[64 - n:])


def test_y_beside_other_memory_is_left_alone():
    c = Layer(3, 36, 20, 6, 2, "fp32").device()
    room = torch.full((5, 36), 9.0, device=DEV)
    c.y = room[1:4]
    c.bind()()
    assert (room[0] == 9.0).all() and (room[4] == 9.0).all()
    c.check(gate=False)


def test_two_shapes_share_a_workspace_and_graphs_replay():
    a, b = Layer(4, 512, 384, 16, 4, F_shared=128).device(), Layer(23, 256, 640, 8, 2, "fp32", act=1).device()
    size = max(a.ws.numel(), b.ws.numel())
    a.ws = b.ws = torch.full((size,), 0x5A, dtype=torch.uint8, device=DEV)
    graphs, wants = [], []
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for c in (a, b):
            call = c.bind()
            call()
            torch.cuda.synchronize()
            wants.append((c.y.clone(), c.idx.clone(), c.w.clone()))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                call(torch.cuda.current_stream().cuda_stream)
            graphs.append(g)
        for i in (0, 1, 1, 0, 1, 0, 0):
            c = (a, b)[i]
            c.y.fill_(float("nan"))
            c.idx.fill_(-7)
            graphs[i].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip((c.y, c.idx, c.w), wants[i]))
            a.bind()()                                                       # eager work between the replays
            torch.cuda.synchronize()


def test_beside_the_step_by_step_path():
    # the same layer by route, dispatch, expert FFN and combine
    c = Layer(16, 512, 384, 8, 2, renorm=1).device()
    c.bind()()
    S = 32
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    idx, w = i32((16, 2)), torch.empty(16, 2, device=DEV)
    P.moe_route(c.ctx, c.d_x, c.d_gate, c.d_bias, idx, w)
    assert torch.equal(idx, c.idx) and torch.allclose(w, c.w, rtol=3e-7, atol=0)
    send, s2r, r2s, so, se = torch.empty(S, 512, dtype=torch.bfloat16, device=DEV), i32(S), i32(S), i32(9), i32(8)
    P.moe_dispatch(c.ctx, c.d_x, idx, [0] * 8, [0], send, s2r, r2s, so, se)
    out, ws = torch.empty_like(send), torch.empty(P.moe_ffn_workspace_bytes(S, 512, 384, 2, "bf16"), dtype=torch.uint8, device=DEV)
    P.moe_expert_ffn(send, S, so, se, 8, c.d_experts, 512, 384, 2, "bf16", out, ws)
    y = torch.empty_like(c.y)
    P.moe_combine(c.ctx, out, s2r, w, None, y)
    H.assert_close(H.host(c.y), H.host(y), "bf16")


def test_a_decode_step_between_two_norms_in_a_graph():
    """norms behind one block and in front of the layer -> layer -> norms behind the layer and in front of the next block, as a decode step replays them."""
    c = Layer(5, 512, 384, 16, 4, F_shared=256).device()
    rng = np.random.default_rng(3)
    some = lambda: dev(on_grid(rng.standard_normal((5, 512)), "bf16"), "bf16")  # noqa: E731
    y0, residual, gamma = some(), some(), dev(on_grid(1 + 0.1 * rng.standard_normal(512), "bf16"), "bf16")
    r1, r2, normed = torch.empty_like(y0), torch.empty_like(y0), torch.empty_like(y0)
    rule = P.block_rule(norm_post=True, gamma_post=gamma, scale=0.5, gamma_pre=gamma)
    calls = [P.bind_block_norm(y0, residual, rule, r1, c.d_x, None), c.bind(), P.bind_block_norm(c.y, r1, rule, r2, normed, None)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for call in calls:
            call(side.cuda_stream)
        side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for call in calls:
                call(torch.cuda.current_stream().cuda_stream)
        gm = gamma.double().cpu().numpy()
        for _ in range(3):
            y0.copy_(some())
            residual.copy_(some())
            for t in (r1, r2, normed, c.d_x, c.y):
                t.fill_(float("nan"))
            g.replay()
            side.synchronize()
            host = lambda t: t.double().cpu().numpy()  # noqa: E731
            assert_rounded(host(r1), B.residual_sum(host(y0), host(residual), gm, None, 0, 0.5, True, 1e-6), "bf16")
            assert_rounded(host(c.d_x), B.normed(host(r1), gm, 1e-6), "bf16")
            c.x = host(c.d_x)
            idx, w, z = O.route(c.x, c.w_gate, c.bias, c.k, c.renorm)
            assert O.route_margin(z, c.k).min() > 1e-9 and np.array_equal(c.idx.cpu().numpy(), idx)
            c.check(gate=False)
            assert_rounded(host(r2), B.residual_sum(host(c.y), host(r1), gm, None, 0, 0.5, True, 1e-6), "bf16")
            assert_rounded(host(normed), B.normed(host(r2), gm, 1e-6), "bf16")


# fp32 widths that end inside 128 bytes and inside 16 rows, in layers of more than 2^18 elements a token, which are no block's work
@pytest.mark.parametrize("T,Hn,F,Fs", [(33, 516, 260, 36), (64, 260, 516, 0), (20, 612, 388, 12), (3, 300, 612, 4), (16, 2052, 36, 0)])
def test_fp32_widths_of_larger_layers(T, Hn, F, Fs):
    for act in range(3):
        Layer(T, Hn, F, 6, 2, "fp32", act, F_shared=Fs, renorm=1).check()


# layers of up to 2^18 elements a token, which a block does, and (the last, and SwiGLU of the sixth) of some more (H, F, E, k, shared)
SMALL = [("fp32", 4, 4, 1, 1, 0), ("fp32", 64, 64, 256, 8, 0), ("fp32", 2048, 4, 3, 2, 20), ("fp32", 16, 2044, 2, 2, 8), ("fp32", 60, 124, 65, 7, 36), ("fp32", 512, 8, 200, 16, 4),
         ("bf16", 128, 128, 8, 2, 128), ("bf16", 128, 128, 3, 3, 0), ("bf16", 256, 128, 64, 1, 128), ("bf16", 640, 128, 5, 1, 0), ("bf16", 1152, 128, 30, 1, 0)]


@pytest.mark.parametrize("T", [1, 5, 64])
@pytest.mark.parametrize("shape", SMALL)
def test_small_layers(shape, T):
    dtype, Hn, F, E, k, Fs = shape
    for act in range(3):
        local = [(e * 7 + 3) % E if e < 64 else -1 for e in range(E)] if E % 7 and E <= 64 else [e if e < 64 else -1 for e in range(E)]
        Layer(T, Hn, F, E, k, dtype, act, local=local, F_shared=Fs, renorm=act % 2, bias=act != 1).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_small_layers_one_by_one_and_with_given_choices(dtype):
    c = Layer(40, 128, 128, 8, 4, dtype, act=1, local=[0, -1, 1, 2, -1, 3, 4, 5], F_shared=128).device()
    c.bind()()
    for n in (1, 3, 17):
        d = Layer(n, 128, 128, 8, 4, dtype, act=1, local=c.local, F_shared=128)
        d.x, d.w_gate, d.bias, d.experts, d.shared = c.x[40 - n:], c.w_gate, c.bias, c.experts, c.shared
        d.device().bind()()
        assert torch.equal(d.y, c.y[40 - n:]) and torch.equal(d.idx, c.idx[40 - n:]) and torch.equal(d.w, c.w[40 - n:])
    before, idx = c.y.clone(), c.idx.clone()
    c.y.fill_(np.nan)
    c.bind(routed=True)()                                                    # its own choices, given
    assert torch.equal(c.y, before)
    c.d_x[2, 3], c.d_x[7, 0] = np.nan, np.inf
    c.bind()()
    keep = [t for t in range(40) if t not in (2, 7)]
    assert c.y[2].isnan().all() and torch.equal(c.y[keep], before[keep]) and torch.equal(c.idx[keep], idx[keep]) and ((c.idx >= 0) & (c.idx < 8)).all()
    c.device()
    rng = np.random.default_rng(3)
    idx = rng.integers(-2, 10, (40, 4)).astype(np.int32)
    idx[4], idx[5], idx[6], idx[7] = -1, 3, [2, 2, 2, 0], [1, 4, 1, 4]       # nobody, one four times, one three times, experts on another GPU
    c.idx.copy_(torch.from_numpy(idx))
    c.w.copy_(torch.from_numpy(rng.random((40, 4)).astype(np.float32)))
    c.bind(routed=True)()
    c.check(gate=False)
    assert np.array_equal(c.idx.cpu().numpy(), idx)
