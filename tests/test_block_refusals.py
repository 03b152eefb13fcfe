"""What the norms around a block refuse and take at their limits (nothing is launched), and the oracle's definitions by hand."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import paper_2410_17043_amd as P
from oracle import block_layer as B
from paper_2410_17043_amd import _lib
from tests.test_oracle_fp8 import A, ODD, status

A2 = C.c_void_p(1 << 21)
bf16, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def rule(**change):
    r = dict(gamma_post=1 << 20, gate=1 << 20, gamma_pre=1 << 20, norm_post=1, gate_rows=2, gate_tokens=2, scale=1.0, eps=1e-6)
    r.update(change)
    return _lib.moe_block_rule(*r.values())


CASES = [
    ("MOE_EINVAL", dict(y=None)), ("MOE_EINVAL", dict(rule=None)), ("MOE_EINVAL", dict(residual_out=None, normed=None, rows=None)), ("MOE_EINVAL", dict(T=-1)),
    ("MOE_EINVAL", dict(H=0)), ("MOE_EINVAL", dict(rule=rule(eps=-1.0))), ("MOE_EINVAL", dict(rule=rule(eps=math.nan))), ("MOE_EINVAL", dict(rule=rule(scale=math.inf))),
    ("MOE_EINVAL", dict(rule=rule(scale=math.nan))), ("MOE_EINVAL", dict(rule=rule(norm_post=2))), ("MOE_EINVAL", dict(rule=rule(norm_post=0))), ("MOE_EDTYPE", dict(dtype=2)),
    ("MOE_EDTYPE", dict(form=2)), ("MOE_ESHAPE", dict(H=32896)), ("MOE_ESHAPE", dict(H=192)), ("MOE_ESHAPE", dict(rule=rule(gate_tokens=1))),
    ("MOE_ESHAPE", dict(rule=rule(gate_rows=0))), ("MOE_ESHAPE", dict(rule=rule(gate_tokens=-2, gate_rows=-2))), ("MOE_EALIGN", dict(H=132, rows=None)), ("MOE_EALIGN", dict(y=ODD)),
    ("MOE_EALIGN", dict(rows=ODD)), ("MOE_EALIGN", dict(rule=rule(gate=(1 << 20) + 8))), ("MOE_EALIGN", dict(rule=rule(gamma_pre=(1 << 20) + 8))), ("MOE_EINVAL", dict(residual_out=A2)),
    ("MOE_OK", dict(T=0)), ("MOE_OK", dict(T=0, y=None, residual_out=None, normed=None, rows=None)), ("MOE_OK", dict(T=0, rule=rule(gate_rows=1, gate_tokens=2 ** 31 - 1))),
]


@pytest.mark.parametrize("want,change", CASES)
def test_block_norm_refusals(want, change):
    lib = _lib.load()
    a = dict(y=A, residual=A, rule=rule(), T=4, H=256, dtype=1, residual_out=A, normed=A2, rows=C.c_void_p(1 << 22), form=1, stream=None)
    a.update(change)
    a["rule"] = None if a["rule"] is None else C.byref(a["rule"])
    rc = lib.moe_block_norm(*a.values())
    assert status(rc) == want and (rc == 0 or b"moe_block_norm" in lib.moe_last_error())


def test_combine_norm_refuses_missing_arrays():
    lib = _lib.load()
    for i in range(4):
        a = [A, A, A, A, None, None, C.byref(rule()), A, A2, None, 0, None]
        a[i] = None
        assert status(lib.moe_combine_norm(*a)) == "MOE_EINVAL" and b"moe_combine_norm" in lib.moe_last_error()


class Ctx:
    """A context's shape without its device memory."""
    def __init__(self, T, H, E, k, dtype):
        self.shape, self.handle, self.lib = _lib.moe_shape(T, H, E, k, 1, dtype, 0, 0), None, _lib.load()


def test_the_binding_checks_arrays_before_their_pointers_are_handed_on():
    e = torch.empty
    y, rows = e(4, 256, dtype=bf16), e(4, P.moe_int8_row_bytes(256), dtype=u8)
    free = P.block_rule()
    good = (y, y, free, y, y, rows, P.ROWS_INT8)
    with pytest.raises(ValueError, match="GPU tensors"):
        P.moe_block_norm(*good)
    for i, wrong in ((1, y.float()), (1, e(3, 256, dtype=bf16)), (3, e(4, 128, dtype=bf16)), (4, y.float()), (5, e(3, 384, dtype=u8)), (5, e(4, 400, dtype=u8)), (5, rows.view(bf16))):
        with pytest.raises(ValueError, match="need"):
            P.moe_block_norm(*good[:i], wrong, *good[i + 1:])
    ctx, ret, s2r, w = Ctx(4, 256, 8, 2, 1), e(8, 256, dtype=bf16), e(8, dtype=i32), e(4, 2, dtype=f32)
    good = (ctx, ret, s2r, w, y, y, free, y, y, rows, P.ROWS_INT8)
    with pytest.raises(ValueError, match="GPU tensors"):
        P.moe_combine_norm(*good)
    for i, wrong in ((1, ret.float()), (1, e(8, 128, dtype=bf16)), (2, e(7, dtype=i32)), (2, s2r.long()), (3, w.double()), (3, e(3, 2, dtype=f32)), (4, e(3, 256, dtype=bf16)),
                     (5, e(3, 256, dtype=bf16)), (9, e(4, 128, dtype=u8))):
        with pytest.raises(ValueError, match="need"):
            P.moe_combine_norm(*good[:i], wrong, *good[i + 1:])


def test_integer_row_bytes():
    assert [P.moe_int8_row_bytes(H) for H in (128, 1152, 2048, 16384)] == [256, 1280, 2176, 16512] == [B.int8_row_bytes(H) for H in (128, 1152, 2048, 16384)]
    assert [P.moe_int8_row_bytes(H) for H in (0, -128, 64, 130)] == [0, 0, 0, 0]


def test_integer_rows_by_hand():
    q, s = B.integer_rows(np.array([[127.0, -0.5, 0.5, 1.5], [0.0, 0.0, 0.0, 0.0], [1.0, math.inf, 0.0, 0.0], [254.0, -254.0, 3.0, 1.0], [1e-44, 0.0, 0.0, 0.0]]))
    assert q.tolist() == [[127, 0, 0, 2], [0] * 4, [0] * 4, [127, -127, 2, 0], [0] * 4]
    assert s[0] == 1.0 and s[1] == 2.0 ** -126 and np.isnan(s[2]) and s[3] == 2.0 and s[4] == 2.0 ** -126


def test_rounding_to_bf16_against_torch():
    v = np.random.default_rng(0).standard_normal(4096) * np.logspace(-20, 20, 4096)
    v = v.astype(np.float32)
    assert np.array_equal(B.round_bf16(v), torch.from_numpy(v).bfloat16().double().numpy())


def test_block_by_hand():
    # 3, 4: mean square 12.5; the gate of the second row is zero
    y, res = np.array([[3.0, 4.0], [1.0, 1.0]]), np.array([[1.0, 1.0], [6.0, 8.0]])
    r = B.residual_sum(y, res, np.array([2.0, 1.0]), np.array([[1.0, 0.5], [0.0, 0.0]]), 1, 2.0, True, 0.0)
    assert np.allclose(r, [[1 + 2 * 2 * 3 / math.sqrt(12.5), 1 + 2 * 0.5 * 4 / math.sqrt(12.5)], [6.0, 8.0]], rtol=1e-15)
    assert np.allclose(B.normed(r, None, 0.0)[1], np.array([6.0, 8.0]) / math.sqrt(50.0), rtol=1e-15)
    ret = np.array([[1.0], [10.0], [100.0]])
    assert B.combine(ret, np.array([[2, -1], [0, 1]]), np.array([[0.5, 1.0], [1.0, 0.25]]), np.array([[1.0], [2.0]])).tolist() == [[51.0], [5.5]]
