"""How the integer FFN runs a share (CPU only: the choice is the host's)."""
import ctypes as C

import numpy as np

from paper_2410_17043_amd import _lib


def plan_of(*args):
    p = (C.c_int32 * 5)()
    lib = _lib.load()
    assert lib.moe_selfcheck_int8_plan(*args, p) == 0, (args, lib.moe_last_error())
    return list(p)


def test_few_rows_stream_the_weights_whatever_their_width():
    # (the e4m3 kernels keep a scale per 128 of K in LDS, which has room for 32768; the integer ones keep none)
    for H, F in ((4096, 32768), (4096, 32896), (2048, 130944), (40960, 8192), (130944, 128), (128, 130944)):
        for R, mt in ((1, 1), (16, 2), (37, 4), (64, 4)):
            for act in range(3):
                assert plan_of(R, 1, 1, H, F, act)[:3] == [mt, 16 * mt, 16 * mt]
    assert plan_of(2000, 1, 1, 4096, 32896, 2)[0] == 0


def test_pieces_fit_and_cover():
    r = np.random.default_rng(61)
    seen = set()
    for _ in range(4000):
        R = int(np.exp(r.uniform(0, np.log(3000))))
        n_used = int(min(R, r.integers(1, 65)))
        nseg = int(min(1024, n_used * r.integers(1, 17)))
        H, F = 128 * int(np.exp(r.uniform(0, np.log(1023)))), 128 * int(np.exp(r.uniform(0, np.log(1023))))
        if H * F < 2 ** 32:
            p = plan_of(R, n_used, nseg, H, F, int(r.integers(0, 3)))
            seen.add((p[0], p[3] > 1, p[4] > 1))
    assert {s[0] for s in seen} == {0, 1, 2, 4} and {s[1:] for s in seen if s[0]} == {(False, False), (False, True), (True, False), (True, True)}


def test_the_choice_is_that_of_the_e4m3_kernels_where_both_stream():
    lib, p = _lib.load(), (C.c_int32 * 5)()
    r = np.random.default_rng(62)
    for _ in range(1000):
        R = int(np.exp(r.uniform(0, np.log(30000))))
        n_used = int(min(R, r.integers(1, 17)))
        args = (R, n_used, n_used, 128 * int(r.integers(1, 65)), 128 * int(r.integers(1, 257)), int(r.integers(0, 3)))
        assert lib.moe_selfcheck_fp8_plan(*args, 256, p) == 0
        assert plan_of(*args)[:3] == list(p)[:3]


def test_refusals():
    lib, p = _lib.load(), (C.c_int32 * 5)()
    for bad in ((0, 1, 1, 128, 128, 0), (5, 6, 6, 128, 128, 0), (5, 2, 1, 128, 128, 0), (5, 1, 1, 100, 128, 0), (5, 1, 1, 128, 131072, 0), (5, 1, 1, 65536, 65536, 0), (5, 1, 1, 128, 128, 3)):
        assert lib.moe_selfcheck_int8_plan(*bad, p) < 0
    assert lib.moe_selfcheck_int8_plan(5, 1, 1, 128, 128, 0, None) < 0
