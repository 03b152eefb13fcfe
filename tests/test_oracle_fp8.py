"""The oracle of the 8-bit share against brute force and hand cases, and the library's refusals (nothing is launched)."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import fp8_layer as O


def test_e4m3_table_and_rounding_against_torch():
    all_bytes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(O.E4M3, all_bytes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    r = np.random.default_rng(0)
    v = np.concatenate([r.uniform(-448, 448, 4000), r.normal(size=4000) * 2.0 ** r.integers(-12, 6, 4000), O.E4M3[:127], -O.E4M3[:127],
                        (O.E4M3[:126] + O.E4M3[1:127]) / 2]).astype(np.float32)
    v = v[np.abs(v) <= 448]
    ref = torch.from_numpy(v).to(torch.float8_e4m3fn)
    assert np.array_equal(O.E4M3[O.e4m3_bytes(v)], ref.double().numpy())


def test_scale_byte_by_its_definition():
    amax = np.array([0.0, 1e-300, 448.0, np.nextafter(448.0, 449), 447.9, 1.0, 2.0 ** -133 * 448, 3.4e38, 896.0])
    b = O.scale_byte(amax)
    for a, v in zip(amax, b):
        assert 1 <= v <= 254 and a <= 448 * 2.0 ** (int(v) - 127)
        assert v == 1 or a > 448 * 2.0 ** (int(v) - 128)
    assert list(b[2:6]) == [127, 128, 127, 119]


def test_blocks_that_are_not_finite_stand_for_nan():
    v = np.ones((2, 256))
    v[0, 3], v[1, 200] = np.inf, np.nan
    q, b = O.quantize_rows(v)
    assert np.all(q[0, :128] == 0x7F) and b[0, 0] == 127 and np.all(np.isnan(O.row_values(q, b)[1, 128:]))
    assert np.all(O.row_values(q, b)[0, 128:] == 1.0) and np.all(O.row_values(q, b)[1, :128] == 1.0)


def test_packed_rows_keep_values_and_pad_with_zeros():
    r = np.random.default_rng(1)
    for H in (128, 1152, 4096):
        q, b = O.quantize_rows(r.normal(size=(3, H)))
        rows = O.pack_rows(q, b)
        assert rows.shape[1] % 128 == 0 and H + H // 128 <= rows.shape[1] < H + H // 128 + 128
        assert np.array_equal(O.unpack_rows(rows, H)[0], q) and np.array_equal(O.unpack_rows(rows, H)[1], b)
        assert not rows[:, H + H // 128:].any()


def test_quantised_values_are_within_half_a_step():
    v = np.random.default_rng(2).normal(size=(16, 512)) * 2.0 ** np.random.default_rng(3).integers(-9, 9, (16, 1))
    d = O.row_values(*O.quantize_rows(v))
    amax = np.repeat(np.abs(v.reshape(16, -1, 128)).max(2), 128, axis=1)
    assert np.all(np.abs(d - v) <= np.maximum(np.abs(v) / 16, amax / 448 * 2 * 2.0 ** -10))


def test_gate_hand_cases():
    logit = lambda p: np.log(np.asarray(p) / (1 - np.asarray(p)))  # noqa: E731
    s = np.array([[0.9, 0.1, 0.6, 0.55, 0.8, 0.05]])
    # groups {0,1} {2,3} {4,5}: by their best 0 and 2 are kept, by the sum of two 1 and 0
    idx, w, _ = O.route_grouped(logit(s), 2, O.SIGMOID, 3, 2, O.GROUP_MAX)
    assert idx.tolist() == [[0, 4]] and np.allclose(w, [[0.9, 0.8]])
    idx, w, _ = O.route_grouped(logit(s), 3, O.SIGMOID, 3, 2, O.GROUP_TOP2, scale=2.0, renorm=1)
    assert idx.tolist() == [[0, 2, 3]] and np.allclose(w, 2 * np.array([[0.9, 0.6, 0.55]]) / 2.05)
    # the bias decides the choice, not the weight
    idx, w, _ = O.route_grouped(logit(s), 1, O.SIGMOID, bias=[0, 0, 0, 0, 0, 2.0])
    assert idx.tolist() == [[5]] and np.allclose(w, [[0.05]])
    # equal scores: lower expert, lower group
    idx, _, _ = O.route_grouped(np.zeros((1, 6)), 2, O.SOFTMAX, 3, 1)
    assert idx.tolist() == [[0, 1]]
    # out of service: fewer than k are left
    idx, w, _ = O.route_grouped(np.zeros((1, 4)), 3, O.SOFTMAX, bias=[-np.inf, 0, -np.inf, -np.inf])
    assert idx.tolist() == [[1, -1, -1]] and w[0, 1] == 0
    # a group with one expert left ranks last where two count
    idx, _, _ = O.route_grouped(logit(s), 2, O.SIGMOID, 3, 2, O.GROUP_TOP2, bias=[0, -np.inf, 0, 0, 0, 0])
    assert idx.tolist() == [[4, 2]]


def test_norm_hand_case():
    r = np.array([[3.0, 4.0, 0.0, 0.0]])
    assert np.allclose(O.norm(r, None, 0.0), r / 2.5)
    assert np.allclose(O.norm(r, [2, 1, 1, 1], 0.0)[0, 0], 2.4)


def test_ffn_against_loops():
    r = np.random.default_rng(4)
    H, F = 128, 256
    w = {}
    for n, shape in (("1", (F, H)), ("_up", (F, H)), ("_down", (H, F))):
        w["w" + n], w["s" + n] = O.quantize_weight(r.normal(size=shape) * 0.1)
    rows = O.pack_rows(*O.quantize_rows(r.normal(size=(3, H))))
    got = O.expert_ffn(rows, H, [0, 2, 2, 3], [0, 0, 5], [w], O.ACT_SWIGLU)
    assert np.all(np.isnan(got[2]))                                          # no such expert
    a = O.row_values(*O.unpack_rows(rows, H))
    for t in range(2):
        h = np.zeros(F)
        for f in range(F):
            g = sum(a[t, k] * O.E4M3[w["w1"][f, k]] * 2.0 ** (int(w["s1"][f // 128, k // 128]) - 127) for k in range(H))
            u = sum(a[t, k] * O.E4M3[w["w_up"][f, k]] * 2.0 ** (int(w["s_up"][f // 128, k // 128]) - 127) for k in range(H))
            h[f] = g / (1 + np.exp(-g)) * u
        hq = O.row_values(*O.quantize_rows(h[None]))[0]
        y = [sum(hq[f] * O.E4M3[w["w_down"][o, f]] * 2.0 ** (int(w["s_down"][o // 128, f // 128]) - 127) for f in range(F)) for o in range(H)]
        assert np.allclose(got[t], y, rtol=1e-12, atol=1e-12)


# ------------------------------------------------------------------------------------------------ refusals
A = C.c_void_p(1 << 20)                    # addresses that are never read: every call below is refused before a launch
ODD = C.c_void_p((1 << 20) + 8)


def status(rc):
    from paper_2410_17043_amd import _lib
    return _lib.load().moe_status_str(rc).decode()


def test_row_bytes():
    import paper_2410_17043_amd as P
    assert [P.moe_fp8_row_bytes(H) for H in (128, 1152, 2048, 4096, 16384)] == [256, 1280, 2176, 4224, 16512]
    assert [P.moe_fp8_row_bytes(H) for H in (0, -128, 64, 130)] == [0, 0, 0, 0]


@pytest.mark.parametrize("want,change", [
    ("MOE_EINVAL", dict(x=None)), ("MOE_EINVAL", dict(residual_out=None, y=None, rows=None)), ("MOE_EINVAL", dict(T=-1)),
    ("MOE_EINVAL", dict(H=0)), ("MOE_EINVAL", dict(eps=-1e-6)), ("MOE_EINVAL", dict(eps=float("nan"))), ("MOE_EINVAL", dict(eps=float("inf"))),
    ("MOE_EDTYPE", dict(dtype=2)), ("MOE_ESHAPE", dict(H=32896)), ("MOE_ESHAPE", dict(H=192)), ("MOE_EALIGN", dict(H=132, rows=None)),
    ("MOE_EALIGN", dict(x=ODD)), ("MOE_EALIGN", dict(gamma=ODD)), ("MOE_EALIGN", dict(rows=ODD)), ("MOE_EINVAL", dict(y=A, residual_out=A)),
    ("MOE_OK", dict(T=0)),
])
def test_norm_refusals(want, change):
    from paper_2410_17043_amd import _lib
    lib = _lib.load()
    a = dict(x=A, residual=None, gamma=A, eps=1e-6, T=4, H=256, dtype=1, residual_out=None, y=A, rows=C.c_void_p(1 << 21), stream=None)
    a.update(change)
    rc = lib.moe_norm_fp8(*a.values())
    assert status(rc) == want and (rc == 0 or b"moe_norm_fp8" in lib.moe_last_error())


@pytest.mark.parametrize("want,change", [
    ("MOE_EINVAL", dict(recv=None)), ("MOE_EINVAL", dict(ws=None)), ("MOE_EINVAL", dict(R=-1)), ("MOE_EINVAL", dict(H=0)), ("MOE_EDTYPE", dict(act=3)),
    ("MOE_ESHAPE", dict(H=192)), ("MOE_ESHAPE", dict(F=1000)), ("MOE_ESHAPE", dict(H=1 << 17, F=1 << 17)), ("MOE_ESHAPE", dict(nseg=1025)),
    ("MOE_ESHAPE", dict(n_local=65)), ("MOE_ESHAPE", dict(n_local=0)), ("MOE_EALIGN", dict(recv=ODD)), ("MOE_EALIGN", dict(out=ODD)), ("MOE_EALIGN", dict(ws=ODD)),
    ("MOE_ESHAPE", dict(bytes=1000)), ("MOE_EINVAL", dict(w_up=None)), ("MOE_EINVAL", dict(s_down=None)), ("MOE_EALIGN", dict(w1=(1 << 20) + 8)),
    ("MOE_OK", dict(R=0)), ("MOE_OK", dict(nseg=0)),
])
def test_ffn_refusals(want, change):
    from paper_2410_17043_amd import _lib
    lib = _lib.load()
    a = dict(recv=A, R=4, so=A, se=A, nseg=1, tab=None, n_local=1, H=256, F=256, act=2, out=A, ws=A, bytes=1 << 30, stream=None)
    tab = (_lib.moe_expert_w8 * 65)()
    for e in tab:
        for n, _ in _lib.moe_expert_w8._fields_:
            setattr(e, n, 1 << 20)
    for n, v in list(change.items()):
        if n in dict(_lib.moe_expert_w8._fields_):
            setattr(tab[0], n, v)
            del change[n]
    a.update(change, tab=tab)
    rc = lib.moe_expert_ffn_fp8(*a.values())
    assert status(rc) == want and (rc == 0 or b"moe_expert_ffn_fp8" in lib.moe_last_error())


def test_ffn_workspace_bytes():
    import paper_2410_17043_amd as P
    for F in (128, 1408, 14336):                                             # a workspace for R_max rows serves any smaller share
        sizes = [P.moe_ffn_fp8_workspace_bytes(R, 256, F, 2) for R in (0, 1, 64, 1000, 1024, 1025, 5000, 100000)]
        assert sizes == sorted(sizes)
    assert P.moe_ffn_fp8_workspace_bytes(100, 256, 384, 2) >= 100 * P.moe_fp8_row_bytes(384)
    for bad in ((-1, 256, 384, 2), (4, 200, 384, 2), (4, 256, 0, 2), (4, 256, 384, 3), (4, 1 << 17, 1 << 17, 2)):
        assert P.moe_ffn_fp8_workspace_bytes(*bad) == 0
