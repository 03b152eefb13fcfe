"""What the 8-bit share refuses and takes at its limits (nothing is launched)."""
import ctypes as C

import pytest

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
