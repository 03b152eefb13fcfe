"""What the 8-bit share refuses and takes at its limits (nothing is launched)."""
import ctypes as C

import pytest
import torch

import paper_2410_17043_amd as P
from paper_2410_17043_amd import _lib
from tests.test_oracle_fp8 import A, status


def ffn_call(**change):
    """moe_expert_ffn_fp8 of no rows with addresses that are never read."""
    a = dict(recv=A, R=0, so=A, se=A, nseg=1, tab=None, n_local=1, H=256, F=256, act=2, out=A, ws=A, bytes=1 << 44, stream=None)
    tab = (_lib.moe_expert_w8 * 1)()
    for n, _ in _lib.moe_expert_w8._fields_:
        setattr(tab[0], n, 1 << 20)
    a.update(change, tab=tab)
    return status(_lib.load().moe_expert_ffn_fp8(*a.values()))


# a tile of 256 rows addresses them by 32-bit offsets: of recv and the intermediate (H or F bytes and scales), of out (2 H bytes)
@pytest.mark.parametrize("H,F,fits", [(8388480, 128, True), (8388608, 128, False), (16777216, 128, False), (256, 16646912, True), (128, 16647040, False)])
def test_ffn_rows_whose_offsets_in_a_tile_pass_32_bits(H, F, fits):
    assert H * F <= 2 ** 32 - 1
    rows = 256 * max(P.moe_fp8_row_bytes(H), P.moe_fp8_row_bytes(F), 2 * H)
    assert (rows <= 2 ** 32 - 256) == fits
    assert (P.moe_ffn_fp8_workspace_bytes(4, H, F, 2) > 0) == fits
    assert ffn_call(H=H, F=F) == ("MOE_OK" if fits else "MOE_ESHAPE")
    if not fits:
        assert b"moe_expert_ffn_fp8" in _lib.load().moe_last_error()


def test_arrays_without_elements_may_be_null():
    # what an empty tensor's pointer is
    lib = _lib.load()
    for dtype in (0, 1):
        assert status(lib.moe_norm_fp8(None, None, A, 1e-6, 0, 256, dtype, None, None, None, None)) == "MOE_OK"
    assert status(lib.moe_norm_fp8(None, None, A, 1e-6, 0, 0, 1, None, None, None, None)) == "MOE_EINVAL"     # the rest is still checked
    assert status(lib.moe_norm_fp8(None, None, A, 1e-6, 4, 256, 1, None, A, None, None)) == "MOE_EINVAL"
    assert ffn_call(recv=None, out=None) == "MOE_OK"
    assert ffn_call(recv=None, out=None, nseg=0, se=None) == "MOE_OK"
    for change in (dict(R=4, recv=None), dict(R=4, out=None), dict(se=None), dict(so=None), dict(ws=None), dict(recv=None, out=None, H=200)):
        assert ffn_call(**change) in ("MOE_EINVAL", "MOE_ESHAPE")


# ------------------------------------------------------------------------------------------------ arrays of the Python binding
class Ctx:
    """A context's shape without its device memory."""
    def __init__(self, T, H, E, k, dtype):
        self.shape, self.handle, self.lib = _lib.moe_shape(T, H, E, k, 1, dtype, 0, 0), None, _lib.load()


def accepted(call, *args):
    """The checks pass: the next thing asked of the arrays is that they lie on the GPU."""
    with pytest.raises(ValueError, match="GPU tensors"):
        call(*args)


bf16, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.mark.parametrize("call", [P.moe_route_grouped, P.bind_route_grouped])
def test_gate_binding_checks_arrays(call):
    ctx = Ctx(4, 256, 24, 3, 1)
    good = dict(x=torch.zeros(4, 256, dtype=bf16), w_gate=torch.zeros(24, 256, dtype=bf16), rule=P.gate_rule(), select_bias=torch.zeros(24),
                topk_idx=torch.zeros(4, 3, dtype=i32), topk_w=torch.zeros(4, 3), workspace=torch.zeros(4096, dtype=u8))
    accepted(call, ctx, *good.values())
    accepted(call, ctx, *dict(good, x=torch.zeros(2, 2, 256, dtype=bf16), select_bias=None).values())         # tokens of two sequences
    accepted(call, ctx, *dict(good, x=torch.zeros(9, 256, dtype=bf16), topk_idx=torch.zeros(12, dtype=i32)).values())   # a longer buffer, a flat one
    for name, t in (("x", torch.zeros(4, 256)), ("x", torch.zeros(3, 256, dtype=bf16)), ("x", torch.zeros(8, 128, dtype=bf16)), ("w_gate", torch.zeros(24, 256)),
                    ("w_gate", torch.zeros(23, 256, dtype=bf16)), ("select_bias", torch.zeros(24, dtype=bf16)), ("select_bias", torch.zeros(23)),
                    ("topk_idx", torch.zeros(4, 3, dtype=torch.int64)), ("topk_idx", torch.zeros(3, 3, dtype=i32)), ("topk_w", torch.zeros(4, 3, dtype=bf16)),
                    ("topk_w", torch.zeros(4, 2))):
        with pytest.raises(ValueError, match="^%s needs" % name):
            call(ctx, *dict(good, **{name: t}).values())


@pytest.mark.parametrize("call", [P.moe_expert_ffn_fp8, P.bind_expert_ffn_fp8])
def test_ffn_binding_checks_arrays(call):
    H, F, R = 1152, 256, 5
    expert = dict(w1=torch.zeros(F, H, dtype=u8), w_up=torch.zeros(F, H, dtype=torch.float8_e4m3fn), w_down=torch.zeros(H, F, dtype=u8), s1=torch.zeros(2, 9, dtype=u8),
                  s_up=torch.zeros(2, 9, dtype=torch.float8_e8m0fnu), s_down=torch.zeros(9, 2, dtype=u8))
    good = dict(recv=torch.zeros(R, 1280, dtype=u8), R=R, seg_offset=torch.zeros(3, dtype=i32), seg_expert=torch.zeros(2, dtype=i32), nseg=2, experts=[expert], H=H, F=F,
                act=P.ACT_SWIGLU, out=torch.zeros(R, H, dtype=bf16), workspace=torch.zeros(4096, dtype=u8))
    accepted(call, *good.values())
    accepted(call, *dict(good, recv=torch.zeros(9, 640, dtype=bf16), seg_offset=torch.zeros(30, dtype=i32)).values())   # the rows of a send buffer
    accepted(call, *dict(good, experts=[dict(expert, w_up=None, s_up=None)], act=P.ACT_SILU_MLP).values())
    for name, t in (("recv", torch.zeros(R, H, dtype=u8)), ("recv", torch.zeros(R, 1161, dtype=u8)), ("recv", torch.zeros(R - 1, 1280, dtype=u8)), ("recv", torch.zeros(R, 1280, dtype=bf16)),
                    ("out", torch.zeros(R, H)), ("out", torch.zeros(R - 1, H, dtype=bf16)), ("seg_offset", torch.zeros(2, dtype=i32)),
                    ("seg_offset", torch.zeros(3, dtype=torch.int64)), ("seg_expert", torch.zeros(1, dtype=i32)), ("seg_expert", torch.zeros(2))):
        with pytest.raises(ValueError, match="^%s needs" % name):
            call(*dict(good, **{name: t}).values())
    for name, t in (("w1", torch.zeros(F, H, dtype=bf16)), ("w1", torch.zeros(F - 128, H, dtype=u8)), ("w_up", torch.zeros(H, F, dtype=u8)), ("w_down", torch.zeros(F, H, dtype=u8)),
                    ("s1", torch.zeros(2, 9)), ("s1", torch.zeros(1, 9, dtype=u8)), ("s_down", torch.zeros(2, 9, dtype=u8))):
        with pytest.raises(ValueError, match="^%s needs" % name):
            call(*dict(good, experts=[dict(expert, **{name: t})]).values())
