"""What the FFN on integer rows and the layer of few tokens refuse and take at their limits (nothing is launched)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2410_17043_amd as P
from paper_2410_17043_amd import _lib
from tests.test_block_refusals import Ctx
from tests.test_oracle_fp8 import A, ODD, status

bf16, f32, i32, i8, u8 = torch.bfloat16, torch.float32, torch.int32, torch.int8, torch.uint8


# ------------------------------------------------------------------------------------------------ integer rows
@pytest.mark.parametrize("want,change", [
    ("MOE_EINVAL", dict(x=None)), ("MOE_EINVAL", dict(rows=None)), ("MOE_EINVAL", dict(T=-1)), ("MOE_EINVAL", dict(H=0)), ("MOE_EDTYPE", dict(dtype=2)), ("MOE_ESHAPE", dict(H=192)),
    ("MOE_ESHAPE", dict(H=131072)), ("MOE_EALIGN", dict(x=ODD)), ("MOE_EALIGN", dict(rows=ODD)), ("MOE_OK", dict(T=0)), ("MOE_OK", dict(T=0, x=None, rows=None))])
def test_quantize_refusals(want, change):
    lib = _lib.load()
    a = dict(x=A, T=4, H=256, dtype=1, rows=C.c_void_p(1 << 21), stream=None)
    a.update(change)
    rc = lib.moe_quantize_int8(*a.values())
    assert status(rc) == want and (rc == 0 or b"moe_quantize_int8" in lib.moe_last_error())


@pytest.mark.parametrize("want,change", [
    ("MOE_EINVAL", dict(recv=None)), ("MOE_EINVAL", dict(out=None)), ("MOE_EINVAL", dict(so=None)), ("MOE_EINVAL", dict(se=None)), ("MOE_EINVAL", dict(ws=None)), ("MOE_EINVAL", dict(R=-1)),
    ("MOE_EINVAL", dict(H=0)), ("MOE_EDTYPE", dict(act=3)), ("MOE_ESHAPE", dict(H=192)), ("MOE_ESHAPE", dict(F=1000)), ("MOE_ESHAPE", dict(H=131072)), ("MOE_ESHAPE", dict(H=130944, F=32896)),
    ("MOE_ESHAPE", dict(nseg=1025)), ("MOE_ESHAPE", dict(n_local=65)), ("MOE_ESHAPE", dict(n_local=0)), ("MOE_EALIGN", dict(recv=ODD)), ("MOE_EALIGN", dict(out=ODD)), ("MOE_EALIGN", dict(ws=ODD)),
    ("MOE_ESHAPE", dict(bytes=1000)), ("MOE_EINVAL", dict(w_up=None)), ("MOE_EINVAL", dict(s_down=None)), ("MOE_EALIGN", dict(w1=(1 << 20) + 8)), ("MOE_EALIGN", dict(s_up=(1 << 20) + 4)),
    ("MOE_OK", dict(R=0)), ("MOE_OK", dict(nseg=0)), ("MOE_OK", dict(R=0, recv=None, out=None)), ("MOE_OK", dict(nseg=0, se=None)), ("MOE_OK", dict(R=0, H=130944, F=32768, bytes=1 << 44))])
def test_ffn_refusals(want, change):
    lib = _lib.load()
    a = dict(recv=A, R=4, so=A, se=A, nseg=1, tab=None, n_local=1, H=256, F=256, act=2, out=A, ws=A, bytes=1 << 30, stream=None)
    tab = (_lib.moe_expert_wi8 * 65)()
    for e in tab:
        for n, _ in _lib.moe_expert_wi8._fields_:
            setattr(e, n, 1 << 20)
    change = dict(change)
    for n in [n for n in change if n in dict(_lib.moe_expert_wi8._fields_)]:
        setattr(tab[0], n, change.pop(n))
    a.update(change, tab=tab)
    rc = lib.moe_expert_ffn_int8(*a.values())
    assert status(rc) == want and (rc == 0 or b"moe_expert_ffn_int8" in lib.moe_last_error())


def test_ffn_workspace_bytes():
    assert P.moe_ffn_int8_workspace_bytes(1000, 256, 512, 2) >= 1000 * (512 * 2 + P.moe_int8_row_bytes(512))
    for R, H, F, act in ((-1, 256, 256, 2), (4, 192, 256, 2), (4, 256, 0, 2), (4, 256, 256, 3), (4, 131072, 256, 2)):
        assert P.moe_ffn_int8_workspace_bytes(R, H, F, act) == 0


def test_the_binding_checks_arrays_of_the_ffn():
    e = torch.empty
    H, F, R = 256, 384, 4
    expert = dict(w1=e(F, H, dtype=i8), w_up=e(F, H, dtype=i8), w_down=e(H, F, dtype=i8), s1=e(F), s_up=e(F), s_down=e(H))
    good = [e(R, P.moe_int8_row_bytes(H), dtype=u8), R, e(3, dtype=i32), e(2, dtype=i32), 2, [expert], H, F, 2, e(R, H, dtype=bf16), e(1 << 20, dtype=u8)]
    with pytest.raises(ValueError, match="GPU tensors"):
        P.moe_expert_ffn_int8(*good)
    wrong = [(0, e(R, 384, dtype=u8)[:3]), (0, e(R, 400, dtype=u8)), (2, e(2, dtype=i32)), (2, e(3, dtype=torch.int64)), (3, e(1, dtype=i32)), (9, e(R, H)), (9, e(3, H, dtype=bf16)),
             (5, [dict(expert, w1=e(F, H, dtype=u8))]), (5, [dict(expert, w_down=e(F, H, dtype=i8))]), (5, [dict(expert, s1=e(H))]), (5, [dict(expert, s_up=e(F, dtype=bf16))])]
    for i, w in wrong:
        with pytest.raises(ValueError, match="needs"):
            P.moe_expert_ffn_int8(*good[:i], w, *good[i + 1:])
    with pytest.raises(ValueError, match="needs"):
        P.moe_quantize_int8(e(4, 256), e(4, 256, dtype=u8))


# ------------------------------------------------------------------------------------------------ layer of few tokens
class FakeCtx(C.Structure):
    """The head of a context, which is all that the checks read."""
    _fields_ = [("s", _lib.moe_shape), ("rest", C.c_void_p * 16)]


def few_call(shape=None, **change):
    s = dict(T=4, H=256, E=8, k=2, G=1, dtype=1, renorm=0, capacity=0)
    s.update(shape or {})
    ctx = FakeCtx(_lib.moe_shape(*s.values()))
    a = dict(ctx=C.byref(ctx), x=A, Wg=A, bias=A, idx=A, w=A, experts=None, n_local=3, local=None, F=256, act=2, shared=None, F_shared=0, y=A, ws=A, bytes=1 << 40, stream=None)
    tab = (_lib.moe_expert_w * 65)()
    for e in tab:
        e.w1 = e.w_up = e.w_down = 1 << 20
    for n in [n for n in change if n in ("w1", "w_up", "w_down")]:
        setattr(tab[1], n, change.pop(n))
    if "experts" not in change:
        change["experts"] = tab
    local = np.array(change.pop("local", [0, -1, 2, 1, -1, -1, -1, -1]), np.int32) if change.get("local", 0) is not None else change.pop("local")
    a.update(change, local=None if local is None else local.ctypes.data_as(C.POINTER(C.c_int32)))
    return _lib.load().moe_layer_few(*a.values())


SHARED = (_lib.moe_expert_w * 1)()
SHARED[0].w1 = SHARED[0].w_up = SHARED[0].w_down = 1 << 20
BAD_SHARED = (_lib.moe_expert_w * 1)()
BAD_SHARED[0].w1 = BAD_SHARED[0].w_down = 1 << 20


@pytest.mark.parametrize("want,change", [
    ("MOE_EINVAL", dict(ctx=None)), ("MOE_EINVAL", dict(x=None)), ("MOE_EINVAL", dict(idx=None)), ("MOE_EINVAL", dict(w=None)), ("MOE_EINVAL", dict(y=None)), ("MOE_EINVAL", dict(ws=None)),
    ("MOE_EINVAL", dict(local=None)), ("MOE_EINVAL", dict(experts=None)), ("MOE_EINVAL", dict(n_local=-1)), ("MOE_EINVAL", dict(F=0)), ("MOE_EINVAL", dict(F_shared=-128)),
    ("MOE_EINVAL", dict(F_shared=128)), ("MOE_EINVAL", dict(shared=SHARED)), ("MOE_EINVAL", dict(Wg=None)), ("MOE_EDTYPE", dict(act=3)), ("MOE_ESHAPE", dict(shape=dict(T=65))),
    ("MOE_ESHAPE", dict(shape=dict(capacity=4))), ("MOE_ESHAPE", dict(n_local=65)), ("MOE_ESHAPE", dict(F=192)), ("MOE_ESHAPE", dict(shape=dict(H=192))),
    ("MOE_ESHAPE", dict(F=262272)), ("MOE_ESHAPE", dict(shape=dict(dtype=0), F=130)), ("MOE_ESHAPE", dict(shared=SHARED, F_shared=64)), ("MOE_EALIGN", dict(x=ODD)), ("MOE_EALIGN", dict(Wg=ODD)),
    ("MOE_EALIGN", dict(y=ODD)), ("MOE_EALIGN", dict(ws=ODD)), ("MOE_ESHAPE", dict(bytes=1000)), ("MOE_ESHAPE", dict(local=[0, 3, -1, -1, -1, -1, -1, -1])),
    ("MOE_ESHAPE", dict(local=[0, -2, -1, -1, -1, -1, -1, -1])), ("MOE_ESHAPE", dict(local=[0, 0, -1, -1, -1, -1, -1, -1])), ("MOE_EINVAL", dict(w1=None)), ("MOE_EINVAL", dict(w_up=None)),
    ("MOE_EALIGN", dict(w_down=(1 << 20) + 8)), ("MOE_EINVAL", dict(shared=BAD_SHARED, F_shared=128))])
def test_layer_few_refusals(want, change):
    rc = few_call(**dict(change))
    assert status(rc) == want and b"moe_layer_few" in _lib.load().moe_last_error()


def test_layer_few_workspace_bytes():
    lib = _lib.load()

    def size(F, F_shared, **change):
        s = dict(T=4, H=256, E=8, k=2, G=1, dtype=1, renorm=0, capacity=0)
        s.update(change)
        ctx = FakeCtx(_lib.moe_shape(*s.values()))
        return int(lib.moe_layer_few_workspace_bytes(C.byref(ctx), F, F_shared))
    assert size(384, 0) >= 4 * 2 * 384 * 2 and size(384, 128) > size(384, 0)
    assert size(384, 0, T=65) == size(192, 0) == size(384, 64) == size(0, 0) == size(262272, 0) == 0 and size(132, 4, dtype=0) > 0
    assert lib.moe_layer_few_workspace_bytes(None, 256, 0) == 0


def test_the_binding_checks_arrays_of_the_layer():
    e = torch.empty
    T, H, E, k, F = 4, 256, 8, 2, 384
    ctx = Ctx(T, H, E, k, 1)
    weights = lambda f: dict(w1=e(f, H, dtype=bf16), w_up=e(f, H, dtype=bf16), w_down=e(H, f, dtype=bf16))  # noqa: E731
    good = [ctx, e(T, H, dtype=bf16), e(E, H, dtype=bf16), e(E), e(T, k, dtype=i32), e(T, k), [weights(F)], [0] + [-1] * 7, F, 2, weights(128), 128, e(T, H, dtype=bf16), e(1 << 20, dtype=u8)]
    with pytest.raises(ValueError, match="GPU tensors"):
        P.moe_layer_few(*good)
    wrong = [(1, e(3, H, dtype=bf16)), (1, e(T, H)), (2, e(E, 128, dtype=bf16)), (3, e(7)), (4, e(T, k, dtype=torch.int64)), (5, e(T, k, dtype=bf16)), (6, [weights(256)]), (6, [dict(weights(F), w1=e(F, H))]),
             (10, weights(256)), (12, e(T, H)), (7, [0] * 7)]
    for i, w in wrong:
        with pytest.raises(ValueError, match="needs"):
            P.moe_layer_few(*good[:i], w, *good[i + 1:])
