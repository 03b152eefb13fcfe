"""How the operators of the 8-bit share choose kernels (host self checks, nothing is launched)."""
import ctypes as C

import numpy as np

from paper_2410_17043_amd import _lib

LDS = 160 * 1024


def gate_plan(T, H, E, n_groups=1, dtype="bf16"):
    p = (C.c_int32 * 4)()
    rc = _lib.load().moe_selfcheck_gate_plan(T, H, E, n_groups, 1 if dtype == "bf16" else 0, p)
    assert rc == 0, ((T, H, E, n_groups, dtype), _lib.load().moe_last_error())
    return dict(zip(("tokens", "pieces", "lds", "limit"), p))


def test_gate_lds_limits_do_not_depend_on_the_launch():
    """A kernel's limit is set once: it has to hold for every launch of that kernel, whichever comes first or at the same time."""
    r = np.random.default_rng(51)
    limits, varies = {}, set()
    for _ in range(3000):
        T, H, E = int(np.exp(r.uniform(0, np.log(40000)))), 8 * int(np.exp(r.uniform(0, np.log(1024)))), int(r.integers(1, 257))
        groups = int(r.choice([g for g in range(1, E + 1) if E % g == 0]))
        p = gate_plan(T, H, E, groups, "bf16" if r.random() < 0.5 else "fp32")
        experts = next(e for e in (16, 32, 64, 128, 256) if E <= e)
        if p["tokens"] == 64:
            experts = max(experts, 32)
        kernel = (p["tokens"], p["pieces"] == 0, experts)
        assert p["lds"] <= p["limit"] == limits.setdefault(kernel, p["limit"]) <= LDS
        if p["lds"] != p["limit"]:
            varies.add(kernel)
    assert varies == {(64, True, 256)}                                       # the logits and the selection's scratch over the ring
    bad = (C.c_int32 * 4)()
    for args in ((0, 128, 8, 1, 1), (4, 128, 8, 3, 1), (4, 128, 300, 1, 1), (4, 100, 8, 1, 1), (4, 128, 8, 1, 2)):
        assert _lib.load().moe_selfcheck_gate_plan(*args, bad) < 0


def test_ffn_tile_maps_of_every_plan_fit_their_records():
    """Both maps and the two records of counters, over shares of every kind; a map of low tiles for many segments alone would not fit, which
    the check has to see."""
    lib, p = _lib.load(), (C.c_int32 * 5)()
    free = lib.moe_selfcheck_fp8_records
    assert free(1100, 1024, 64, 64) == -2 and free(1100, 1024, 128, 128) == 7 and free(1100, 1024, 64, 128) < -1000 and free(1024, 1024, 16, 16) == 15
    r = np.random.default_rng(52)
    low = 10 ** 9
    for _ in range(6000):
        R = int(np.exp(r.uniform(0, np.log(200000))))
        n_used = int(min(R, r.integers(1, 65)))
        nseg = int(r.choice([n_used, min(1024, n_used * int(r.integers(1, 17))), 1024]))
        H, F = 128 * int(np.exp(r.uniform(0, np.log(64)))), 128 * int(np.exp(r.uniform(0, np.log(300))))
        args = (R, n_used, nseg, H, F, int(r.integers(0, 3)), 256)
        assert lib.moe_selfcheck_fp8_plan(*args, p) == 0, (args, lib.moe_last_error())
        low = min(low, free(R, nseg, p[1], p[2]))
        assert free(R, nseg, p[1], p[2]) >= 0
    assert low < 20                                                          # the tight ones were among them
    for bad in ((0, 4, 64, 64), (4, 0, 64, 64), (4, 1025, 64, 64), (4, 4, 0, 64), (4, 4, 64, 512)):
        assert free(*bad) == -(1 << 30)
