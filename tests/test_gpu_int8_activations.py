"""Every epilogue of the integer FFN's first product at arguments where the activations differ from each other and from their argument.

Against the oracle in 64 bits, with the bounds of tests/test_gpu_int8.py for ordinary weights; that another activation is ten times outside of them is asserted beside each."""
import numpy as np
import pytest

from oracle import block_layer as B
from tests import harness as H
from tests.test_gpu_int8 import GELU, SILU, SWIGLU, make_experts, make_rows, on_device, plan_of, run_ffn, to_dev

pytestmark = pytest.mark.gpu


def check(R, Hn, F, act, n_local):
    r = np.random.default_rng([R, Hn, F, act])
    so = [R * i // n_local for i in range(n_local + 1)]
    q, s = make_rows(r, R, Hn, False)
    experts = make_experts(r, n_local, Hn, F, act, False)
    out = run_ffn(to_dev(B.pack_integer_rows(q, s)), so, list(range(n_local)), on_device(experts), Hn, F, act).double().cpu().numpy()
    want = np.concatenate([B.expert_ffn_int8(q[a:b], s[a:b], e, act) for a, b, e in zip(so, so[1:], experts)])
    H.assert_close(out, want, "bf16")
    some = slice(so[0], min(so[1], 20))
    e = dict(experts[0])
    if act == SWIGLU:                                                        # gate and up in each other's place
        e["w1"], e["w_up"], e["s1"], e["s_up"] = e["w_up"], e["w1"], e["s_up"], e["s1"]
    other = B.expert_ffn_int8(q[some], s[some], e, {SILU: GELU, GELU: SILU, SWIGLU: SWIGLU}[act])
    assert H.rms_rel_err(other, want[some]) > 10 * H.RMS_TOL["bf16"]


def columns(R, n_local, mt, N):
    """of a block that streams the weights: 64 where such blocks are at most 256."""
    return 64 if (R + n_local * (16 * mt - 1)) // (16 * mt) * (N // 64) <= 256 else 128


# rows of a tile / 16, columns of a block of the first and of the second product
@pytest.mark.parametrize("act,R,n_local,Hn,F,mt,first,second", [(act,) + c for c in [
    (3, 1, 256, 640, 1, 64, 64), (200, 8, 896, 640, 1, 64, 128), (200, 24, 512, 640, 1, 128, 128),
    (400, 4, 1152, 640, 2, 64, 128), (400, 24, 512, 640, 2, 128, 128),
    (40, 1, 256, 4096, 4, 64, 64), (400, 16, 1152, 640, 4, 64, 128)] for act in (SILU, GELU, SWIGLU)] + [(act,) + c for c in [
        (20, 1, 256, 2304, 2, 64, 64), (400, 2, 256, 640, 1, 128, 64), (400, 16, 256, 640, 2, 128, 64), (800, 16, 256, 640, 4, 128, 64), (800, 24, 512, 640, 4, 128, 128)] for act in (SILU, GELU)] + [
    (SWIGLU, 20, 1, 256, 4096, 2, 64, 64), (SWIGLU, 200, 8, 256, 1408, 2, 128, 64), (SWIGLU, 200, 2, 256, 4096, 4, 128, 64), (SWIGLU, 400, 4, 2048, 2304, 4, 128, 128)])
def test_streamed(act, R, n_local, Hn, F, mt, first, second):
    assert plan_of(R, n_local, n_local, Hn, F, act)["mt"] == mt
    assert (columns(R, n_local, mt, F), columns(R, n_local, mt, Hn)) == (first, second)
    check(R, Hn, F, act, n_local)


@pytest.mark.parametrize("act,R,n_local,Hn,F,want", [(act,) + c for c in [
    (1200, 1, 128, 256, dict(bm1=128, bm2=128, deep=1)), (9000, 1, 512, 256, dict(bm1=128, bm2=128, deep=0)),
    (6000, 2, 512, 2304, dict(bm1=256, bm2=128)), (9000, 1, 1024, 1408, dict(bm1=256, bm2=256))] for act in (SILU, GELU)] + [
    (SWIGLU, 1200, 1, 128, 256, dict(bm1=64, bm2=128)), (SWIGLU, 9000, 1, 512, 256, dict(bm1=128)), (SWIGLU, 9000, 1, 512, 1408, dict(bm1=256, bm2=128)),
    (SWIGLU, 9000, 1, 1024, 640, dict(bm1=256, bm2=256))])
def test_in_tiles(act, R, n_local, Hn, F, want):
    plan = plan_of(R, n_local, n_local, Hn, F, act)
    assert plan["mt"] == 0 and {k: plan[k] for k in want} == want, plan
    check(R, Hn, F, act, n_local)
