"""The intermediate of the 8-bit FFN, byte by byte.

Exactly: every weight row has one element that is not zero, so all sums are exact; the activations return a large argument itself, bit for bit; and the second
product hands single elements of the quantised intermediate on.  What comes out has to equal the definition: no tolerance.  A scale byte that is one too large,
a tie that goes the wrong way, an operand that loses a bit or a column that lands beside its place changes it.

With ordinary weights, for shares of few rows, which stream the weights: products are exact and sums fp32, so an element is what the exact one rounds to unless that
lies within the sums' error of the middle of two e4m3 numbers.  The error: an operand's K / 32 partial sums are rounded to 2^-24 each; of K = 2048 products p of either sign,
partial sums stay near sqrt(K) of a product where the sum of |p| is near K of them, so 64 roundings come to 1e-8 of the sum of |p| (in the 2-norm); 2^-23, twelve times that, is
allowed, and 1e-6 of the activation.  (The matrix cores' own e4m3 products, in the tiles of larger shares, are off by 5e-7 of the sum of |p|.)"""
import numpy as np
import pytest

from oracle import fp8_layer as O
from tests import harness as H
from tests.test_gpu_fp8 import experts_to_dev, make_experts, make_rows, plan_of, run_ffn8

pytestmark = pytest.mark.gpu


def one_per_row(r, n, K, first_column, negative):
    """e4m3 [n, K] with one positive number (of either sign, if negative) per row, from `first_column` on."""
    w = np.zeros((n, K), dtype=np.uint8)
    sign = np.where(r.random(n) < 0.5, 0x80, 0).astype(np.uint8) if negative else 0
    w[np.arange(n), r.integers(first_column, K, n)] = r.integers(0x01, 0x7F, n).astype(np.uint8) | sign
    return w


def make(r, R, Hn, F, act, n_experts):
    q = r.integers(0x01, 0x7F, (R, Hn)).astype(np.uint8)                     # 2^-9 .. 448
    q[r.random((R, Hn)) < 0.05] = 0
    q[:, 0] = 0x68                                                           # 64: SwiGLU's gate
    b = np.full((R, Hn // 128), 127)
    if act != O.ACT_SWIGLU:                                                  # arguments of at least 2^22, or zero
        b[:] = 147
    rows = O.pack_rows(q, b)
    experts = []
    for _ in range(n_experts):
        e = dict(w_up=None, s_up=None, s1=np.full((F // 128, Hn // 128), 147 if act != O.ACT_SWIGLU else 127, dtype=np.uint8), s_down=np.full((Hn // 128, F // 128), 127, dtype=np.uint8))
        if act == O.ACT_SWIGLU:
            e["w1"] = np.zeros((F, Hn), dtype=np.uint8)
            e["w1"][:, 0] = 0x38                                             # 1
            e["w_up"], e["s_up"] = one_per_row(r, F, Hn, 1, True), r.integers(100, 150, (F // 128, Hn // 128)).astype(np.uint8)
        else:
            e["w1"] = one_per_row(r, F, Hn, 1, False)
        e["w_down"] = np.zeros((Hn, F), dtype=np.uint8)
        take = np.concatenate([r.permutation(F) for _ in range(-(-Hn // F))])[:Hn]
        e["w_down"][np.arange(Hn), take] = 0x38
        experts.append(e)
    return rows, experts


def intermediate(rows, e, Hn, act):
    a = O.row_values(*O.unpack_rows(rows, Hn))
    return O.activation(act, a @ O.weight_values(e["w1"], e["s1"]).T, a @ O.weight_values(e["w_up"], e["s_up"]).T if act == O.ACT_SWIGLU else None)


def what_is_met(h):
    """Blocks whose largest element is 448 times a power of two, blocks just above; ties among normal and among subnormal results."""
    blocks = h.reshape(len(h), -1, 128)
    amax = np.abs(blocks).max(2)
    b = O.scale_byte(amax)
    unit = np.ldexp(1.0, b - 127)
    t = np.abs(blocks) / unit[..., None]
    hi = np.clip(np.searchsorted(O._POSITIVE, t), 1, 126)
    tie = (t > 0) & (t - O._POSITIVE[hi - 1] == O._POSITIVE[hi] - t)
    return (amax == 448 * unit).sum(), ((amax > 224 * unit) & (amax < 232 * unit)).sum(), (tie & (t > 2.0 ** -6)).sum(), (tie & (t < 2.0 ** -6)).sum()


@pytest.mark.parametrize("R,Hn,F,act,n_local,want", [
    (5, 1024, 8192, O.ACT_SWIGLU, 1, dict(mt=1)), (20, 1024, 8192, O.ACT_GELU_MLP, 1, dict(mt=2)), (60, 896, 8064, O.ACT_SWIGLU, 1, dict(mt=4)),
    (100, 256, 4096, O.ACT_SILU_MLP, 2, dict(mt=4)), (403, 2048, 1408, O.ACT_SWIGLU, 4, dict(mt=2)),
    (1200, 512, 640, O.ACT_SWIGLU, 3, dict(mt=0, bm1=64, bm2=128, deep=1)), (3000, 512, 1408, O.ACT_SWIGLU, 1, dict(mt=0, bm1=128, bm2=128)),
    (9000, 384, 1408, O.ACT_SWIGLU, 2, dict(mt=0, bm1=256)), (9000, 256, 2304, O.ACT_SILU_MLP, 2, dict(mt=0, bm1=128)), (9000, 256, 2304, O.ACT_GELU_MLP, 2, dict(mt=0, bm1=128)),
    (6000, 2048, 2304, O.ACT_SILU_MLP, 1, dict(mt=0, bm1=256, bm2=256)), (6000, 2048, 2304, O.ACT_GELU_MLP, 1, dict(mt=0, bm1=256, bm2=256)),
    (1100, 128, 14336, O.ACT_GELU_MLP, 1, dict(mt=0, bm2=256, pieces=7))])
def test_ffn_intermediate_is_quantised_exactly(R, Hn, F, act, n_local, want):
    r = np.random.default_rng(R + F)
    plan = plan_of(R, n_local, n_local, Hn, F, act)
    assert {k: plan[k] for k in want} == want, plan
    rows, experts = make(r, R, Hn, F, act, n_local)
    so = [R * i // n_local for i in range(n_local + 1)]
    some = np.unique(np.concatenate([r.integers(0, R, 150), so[:-1], np.array(so[1:]) - 1]))       # the rows that are compared
    met = np.zeros(4, dtype=int)
    out = H.host(run_ffn8(rows, so, list(range(n_local)), experts_to_dev(experts), Hn, F, act)).astype(np.float64)
    for e in range(n_local):
        mine = some[(some >= so[e]) & (some < so[e + 1])]
        h = intermediate(rows[mine], experts[e], Hn, act)
        met += what_is_met(h)
        value = O.row_values(*O.quantize_rows(h))
        assert np.array_equal(out[mine], value[:, experts[e]["w_down"].argmax(1)])
    assert np.all(met > 0), met


@pytest.mark.parametrize("R,row_byte,up_byte", [(20, 3, 246), (60, 3, 200), (20, 246, 3), (60, 200, 3), (1100, 3, 246), (1100, 246, 3)])
def test_scales_at_the_ends_of_their_range(R, row_byte, up_byte):
    """Rows of 2^-133 to 2^-115 with weights of up to 2^128, and the other way round: products of ordinary size, from operands that bf16 and fp32 hold as subnormal numbers."""
    Hn, F, act = 256, 512, O.ACT_SWIGLU
    r = np.random.default_rng(R + row_byte)
    assert (plan_of(R, 1, 1, Hn, F, act)["mt"] > 0) == (R <= 1024)
    rows, experts = make(r, R, Hn, F, act, 1)
    rows[:, Hn + 1] = row_byte                                               # the first block holds the gate's 64
    e = experts[0]
    e["w_up"], e["s_up"] = one_per_row(r, F, Hn, 128, True), np.full((F // 128, Hn // 128), up_byte, dtype=np.uint8)
    out = H.host(run_ffn8(rows, [0, R], [0], experts_to_dev(experts), Hn, F, act)).astype(np.float64)
    h = intermediate(rows, e, Hn, act)
    assert np.array_equal(out, O.row_values(*O.quantize_rows(h))[:, e["w_down"].argmax(1)])


@pytest.mark.parametrize("act", [O.ACT_SILU_MLP, O.ACT_GELU_MLP, O.ACT_SWIGLU])
@pytest.mark.parametrize("Hn,F", [(128, 128), (256, 128), (128, 384), (384, 640), (1152, 256), (256, 1408)])
def test_ffn_tiles_with_few_rows_in_them(Hn, F, act):
    """Shares that do not stream: experts of 1 to 129 rows beside a large one, in segments that are not adjacent, empty ones and experts that do not exist."""
    seg_rows, seg_expert, n_local = [900, 1, 0, 5, 64, 7, 33, 129, 31, 2, 300], [0, 1, 2, 3, 4, 9, 5, 6, 5, 3, 0], 8
    r = np.random.default_rng(Hn + F + act)
    so = np.concatenate([[2], 2 + np.cumsum(seg_rows)])                      # two rows in front and three behind belong to no segment
    R = int(so[-1]) + 3
    assert plan_of(R, n_local, len(seg_rows), Hn, F, act)["mt"] == 0
    rows, experts = make(r, R, Hn, F, act, n_local)
    out = H.host(run_ffn8(rows, so, seg_expert, experts_to_dev(experts), Hn, F, act)).astype(np.float64)
    want = np.full((R, Hn), np.nan)
    for e, lo, hi in zip(seg_expert, so[:-1], so[1:]):
        if e < n_local and hi > lo:
            want[lo:hi] = O.row_values(*O.quantize_rows(intermediate(rows[lo:hi], experts[e], Hn, act)))[:, experts[e]["w_down"].argmax(1)]
    assert np.array_equal(out, want, equal_nan=True)


def one_of_both(r, R, Hn, F, act):
    """Rows and weights of every size, an expert whose second product hands the intermediate on."""
    e = make_experts(r, 1, Hn, F, act)[0]
    e["s_down"][:] = 127
    e["w_down"][:] = 0
    take = np.concatenate([r.permutation(F) for _ in range(-(-Hn // F))])[:Hn]
    e["w_down"][np.arange(Hn), take] = 0x38
    return make_rows(r, R, Hn), e, take


@pytest.mark.parametrize("R,Hn,F,act,mt", [(9, 2048, 8192, O.ACT_SWIGLU, 1), (12, 2048, 8192, O.ACT_GELU_MLP, 1), (25, 2048, 8192, O.ACT_SILU_MLP, 2), (26, 2048, 8192, O.ACT_SWIGLU, 2),
                                           (64, 2048, 8192, O.ACT_SWIGLU, 4), (60, 2048, 8192, O.ACT_GELU_MLP, 4)])
def test_few_rows_round_the_exact_intermediate(R, Hn, F, act, mt):
    r = np.random.default_rng(R + mt)
    assert plan_of(R, 1, 1, Hn, F, act)["mt"] == mt
    rows, e, take = one_of_both(r, R, Hn, F, act)
    out = H.host(run_ffn8(rows, [0, R], [0], experts_to_dev([e]), Hn, F, act)).astype(np.float64)
    a, w1 = O.row_values(*O.unpack_rows(rows, Hn)), O.weight_values(e["w1"], e["s1"])
    g, dg = a @ w1.T, 2.0 ** -23 * (np.abs(a) @ np.abs(w1).T)
    h = O.activation(act, g, 1.0)
    dh = 1.2 * dg + 1e-6 * np.abs(h)                                         # the activations' slopes are at most 1.13
    if act == O.ACT_SWIGLU:
        w_up = O.weight_values(e["w_up"], e["s_up"])
        u, du = a @ w_up.T, 2.0 ** -23 * (np.abs(a) @ np.abs(w_up).T)
        h, dh = h * u, dh * np.abs(u) + np.abs(h) * du + dh * du
    amax = np.abs(h).reshape(R, -1, 128).max(2)
    worst = dh.reshape(R, -1, 128).max(2)
    b = O.scale_byte(amax)
    sure = (O.scale_byte(np.maximum(amax - worst, 0)) == b) & (O.scale_byte(amax + worst) == b)
    assert sure.mean() > 0.99
    unit, sure = np.repeat(np.ldexp(1.0, b - 127), 128, 1), np.repeat(sure, 128, 1)
    least, most = (O.E4M3[O.e4m3_bytes(np.clip(v / unit, -448, 448))] * unit for v in (h - dh, h + dh))
    assert (least == most)[sure].mean() > 0.99                               # hardly any element is left to chance
    assert np.all(((least[:, take] <= out) & (out <= most[:, take])) | ~sure[:, take])
