"""Bounds shared by the tests of what surrounds a block and of 8-bit integer rows.

What the kernels form in 64 bits and round once has to be a nearest number of its format to the oracle's 64-bit value, whose own arithmetic (sums of up to 32768
terms, a root, a few products) is off by at most some 1e-12 of a row's largest value."""
import numpy as np
import torch

from oracle import block_layer as B
from oracle import fp8_layer as F8

WIDE = 1e-11


def on_grid(v, dtype):
    """float64 values on the grid of bf16 or fp32."""
    t = torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32))
    return (t.bfloat16() if dtype == "bf16" else t).double().numpy()


def nearest(v, dtype):
    """Rounded once, subnormal numbers and overflows of fp32 aside."""
    return B.round_bf16(v) if dtype == "bf16" else np.asarray(v, np.float64).astype(np.float32).astype(np.float64)


def assert_rounded(got, exact, dtype):
    got, exact = np.asarray(got, np.float64), np.asarray(exact, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(exact))
    fine = np.isfinite(exact) & (np.abs(exact) < 3e38)
    assert np.array_equal(got[~fine & ~np.isnan(exact)], np.sign(exact[~fine & ~np.isnan(exact)]) * np.inf) or not (~fine).any()
    g, e = got[fine], exact[fine]
    slack = WIDE * np.broadcast_to(np.max(np.abs(np.where(np.isfinite(exact), exact, 0.0)), axis=1, keepdims=True), exact.shape)[fine] + 1e-39
    assert np.all(np.abs(g - e) <= np.abs(nearest(e, dtype) - e) + slack)


def assert_integer_rows(rows, v):
    """Packed integer rows (host bytes) hold v."""
    H = v.shape[1]
    q, s = rows[:, :H].view(np.int8).astype(np.float64), np.ascontiguousarray(rows[:, H:H + 4]).view(np.float32).astype(np.float64)[:, 0]
    assert not rows[:, H + 4:].any()                                           # padding
    want = B.integer_scale(v)
    assert np.array_equal(np.isnan(s), np.isnan(want))
    fine = np.isfinite(want)
    assert not q[~fine].any()
    assert np.all(np.abs(s[fine] - want[fine]) <= 2.0 ** -23 * want[fine] * (np.abs(s[fine] - want[fine]) > 0))
    assert np.mean(s[fine] != want[fine]) <= 1e-3                               # the next number only where the 64-bit quotient lies at the middle of two
    assert np.all(np.abs(q[fine] - v[fine] / s[fine, None]) <= 0.5 + 127 * 1e-9)


def assert_e4m3_rows(rows, v):
    H = v.shape[1]
    q, b = F8.unpack_rows(rows, H)
    assert not rows[:, H + H // 128:].any()
    blocks = v.reshape(v.shape[0], -1, 128)
    amax = np.abs(blocks).max(2)
    bad = ~np.isfinite(amax) | (amax > 3.4e38)
    fine = np.where(bad, 0.0, amax)
    assert np.all((F8.scale_byte(fine * (1 - WIDE)) <= b) & (b <= F8.scale_byte(fine * (1 + WIDE))) | (bad & (b == 127)))
    got = F8.E4M3[q].reshape(blocks.shape)
    assert np.array_equal(np.isnan(got), np.broadcast_to(bad[..., None], got.shape))
    t = np.where(bad[..., None], 0.0, blocks) / np.ldexp(1.0, b.astype(int) - 127)[..., None]
    step = np.ldexp(1.0, np.maximum(np.floor(np.log2(np.maximum(np.abs(t), 1e-300))), -6).astype(int) - 3)
    assert np.all(np.abs(np.where(bad[..., None], 0.0, got) - t) <= step / 2 + 448 * WIDE)
