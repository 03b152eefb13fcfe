"""The intermediate of the 8-bit FFN, byte by byte.  Every weight row has one element that is not zero, so all sums are exact; the activations return a
large argument itself, bit for bit; and the second product hands single elements of the quantised intermediate on.  What comes out has to equal the definition:
no tolerance.  A scale byte that is one too large, a tie that goes the wrong way or a column that lands beside its place changes it.

(With ordinary weights none of this shows: the first product's sums are off by up to 1.5e-5, an element that lies that near to the middle of two e4m3 numbers may go
to the other, and `out` is then 0.0018 to 0.0028 off in the 2-norm where rounding it to bf16 alone gives 0.0017.)"""
import numpy as np
import pytest

from oracle import fp8_layer as O
from tests import harness as H
from tests.test_gpu_fp8 import experts_to_dev, plan_of, run_ffn8

pytestmark = pytest.mark.gpu


def one_per_row(r, n, K, first_column, negative):
    """e4m3 [n, K] with one normal number per row, from `first_column` on."""
    w = np.zeros((n, K), dtype=np.uint8)
    sign = np.where(r.random(n) < 0.5, 0x80, 0).astype(np.uint8) if negative else 0
    w[np.arange(n), r.integers(first_column, K, n)] = r.integers(0x08, 0x7F, n).astype(np.uint8) | sign
    return w


def make(r, R, Hn, F, act, n_experts):
    q = r.integers(0x08, 0x7F, (R, Hn)).astype(np.uint8)                     # 2^-6 .. 448
    q[r.random((R, Hn)) < 0.05] = 0
    q[:, 0] = 0x68                                                           # 64: SwiGLU's gate
    b = np.full((R, Hn // 128), 127)
    if act != O.ACT_SWIGLU:                                                  # arguments of at least 2^8, or zero
        b[:] = 137
    rows = O.pack_rows(q, b)
    experts = []
    for _ in range(n_experts):
        e = dict(w_up=None, s_up=None, s1=np.full((F // 128, Hn // 128), 137 if act != O.ACT_SWIGLU else 127, dtype=np.uint8), s_down=np.full((Hn // 128, F // 128), 127, dtype=np.uint8))
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
