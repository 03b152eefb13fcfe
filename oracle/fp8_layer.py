"""The 8-bit form of a layer share in fp64 (numpy), from the definitions in include/aurora_moe.h: quantisation, packed rows,
norm, gate with groups, expert FFN."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 128
SOFTMAX, SIGMOID = 0, 1
GROUP_MAX, GROUP_TOP2 = 0, 1
ACT_SILU_MLP, ACT_GELU_MLP, ACT_SWIGLU = 0, 1, 2


def _e4m3_table():
    v = np.full(256, np.nan)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        if (b & 127) != 127:
            v[b] = (-1.0 if b & 128 else 1.0) * (math.ldexp(1 + m / 8, e - 7) if e else math.ldexp(m / 8, -6))
    return v


E4M3 = _e4m3_table()                       # value of every byte
_POSITIVE = E4M3[:127]                     # ascending: 0 .. 448


def e4m3_bytes(v):
    """Nearest e4m3 byte, ties to the even mantissa; |v| <= 448 (or NaN)."""
    v = np.asarray(v, dtype=np.float64)
    a = np.where(np.isnan(v), 0.0, np.abs(v))
    assert np.all(a <= 464.0), a.max()
    hi = np.clip(np.searchsorted(_POSITIVE, a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - _POSITIVE[lo], _POSITIVE[hi] - a
    take_hi = (above < below) | ((above == below) & (hi % 2 == 0))
    b = np.where(take_hi, hi, lo).astype(np.uint8) | np.where(np.signbit(v), 0x80, 0).astype(np.uint8)
    return np.where(np.isnan(v), np.uint8(0x7F), b).astype(np.uint8)


def scale_byte(amax):
    """Smallest b >= 1 with amax <= 448 * 2^(b - 127); amax finite."""
    amax = np.asarray(amax, dtype=np.float64)
    b = np.ones(amax.shape, dtype=np.int64)
    for k in range(2, 255):
        b = np.where(amax > 448.0 * math.ldexp(1.0, k - 1 - 127), k, b)
    return b


def quantize(v, axes_blocks):
    """v in blocks -> (bytes, scale bytes); `axes_blocks`: the axes of a block."""
    amax = np.max(np.abs(v), axis=axes_blocks, keepdims=True)
    bad = ~np.isfinite(amax)
    b = np.where(bad, 127, scale_byte(np.where(bad, 0.0, amax)))
    with np.errstate(invalid="ignore"):
        t = np.where(bad, np.nan, v / np.ldexp(1.0, b - 127))
    return e4m3_bytes(t), np.squeeze(b, axes_blocks).astype(np.uint8)


def quantize_rows(v):
    """[n, K] -> bytes [n, K], scale bytes [n, K / 128]."""
    v = np.asarray(v, dtype=np.float64)
    q, b = quantize(v.reshape(v.shape[0], -1, BLOCK), (2,))
    return q.reshape(v.shape), b


def row_values(q, b):
    return E4M3[q] * np.repeat(np.ldexp(1.0, b.astype(np.int64) - 127), BLOCK, axis=1)


def row_bytes(H):
    return -(-(H + H // BLOCK) // 128) * 128


def pack_rows(q, b):
    n, H = q.shape
    out = np.zeros((n, row_bytes(H)), dtype=np.uint8)
    out[:, :H] = q
    out[:, H:H + H // BLOCK] = b
    return out


def unpack_rows(rows, H):
    return rows[:, :H], rows[:, H:H + H // BLOCK]


def quantize_weight(w):
    """[n, K] -> bytes [n, K], scale bytes [n / 128, K / 128]."""
    w = np.asarray(w, dtype=np.float64)
    n, K = w.shape
    q, b = quantize(w.reshape(n // BLOCK, BLOCK, K // BLOCK, BLOCK), (1, 3))
    return q.reshape(n, K), b


def weight_values(q, b):
    s = np.ldexp(1.0, b.astype(np.int64) - 127)
    return E4M3[q] * np.repeat(np.repeat(s, BLOCK, axis=0), BLOCK, axis=1)


def norm(r, gamma, eps):
    """v of the definition for r = x (+ residual), already rounded to its type."""
    r = np.asarray(r, dtype=np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        v = r / np.sqrt(np.mean(r * r, axis=1, keepdims=True) + eps)
    return v if gamma is None else v * np.asarray(gamma, dtype=np.float64)


def selection(logits, score, bias):
    """(selection scores with -inf for what is never chosen, scores)."""
    with np.errstate(all="ignore"):
        if score == SOFTMAX:
            p = np.exp(logits - np.max(logits, axis=1, keepdims=True))
            s = p / np.sum(p, axis=1, keepdims=True)
        else:
            s = 1.0 / (1.0 + np.exp(-logits))
        c = s if bias is None else s + np.asarray(bias, dtype=np.float64)
    return np.where(np.isnan(c), -np.inf, c), s


def group_ranks(c, n_groups, group_rank):
    T, E = c.shape
    g = np.sort(c.reshape(T, n_groups, E // n_groups), axis=2)[:, :, ::-1]
    if group_rank == GROUP_MAX or E // n_groups == 1:
        return g[:, :, 0]
    with np.errstate(invalid="ignore"):
        r = g[:, :, 0] + g[:, :, 1]
    return np.where(np.isnan(r), -np.inf, r)


def route_grouped(logits, k, score, n_groups=1, top_groups=1, group_rank=GROUP_MAX, scale=1.0, bias=None, renorm=0):
    """Token by token: kept groups, then k extractions.  Returns (indices, weights, smallest gap that decided)."""
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    c, s = selection(logits, score, bias)
    ranks = group_ranks(c, n_groups, group_rank)
    idx, w = np.full((T, k), -1, dtype=np.int64), np.zeros((T, k))
    gap = np.full(T, np.inf)
    for t in range(T):
        groups = sorted(range(n_groups), key=lambda g: (-ranks[t, g], g))
        if top_groups < n_groups and np.isfinite(ranks[t, groups[top_groups]]):
            gap[t] = min(gap[t], ranks[t, groups[top_groups - 1]] - ranks[t, groups[top_groups]])
        allowed = set(groups[:top_groups])
        experts = sorted((e for e in range(E) if e // (E // n_groups) in allowed and c[t, e] > -np.inf), key=lambda e: (-c[t, e], e))
        for j, e in enumerate(experts[:k]):
            idx[t, j], w[t, j] = e, s[t, e]
            if j + 1 < len(experts):
                gap[t] = min(gap[t], c[t, e] - c[t, experts[j + 1]])
    if renorm:
        total = w.sum(1, keepdims=True)
        w = np.divide(w, total, out=np.zeros_like(w), where=total > 0)
    return idx, w * scale, gap


def activation(act, a, b):
    with np.errstate(over="ignore", invalid="ignore"):
        if act == ACT_GELU_MLP:
            return 0.5 * a * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (a + 0.044715 * a ** 3)))
        return a / (1.0 + np.exp(-a)) * (b if act == ACT_SWIGLU else 1.0)


def expert_ffn(rows, H, seg_offset, seg_expert, experts, act):
    """rows: packed rows; experts: dicts of bytes w1, w_up, w_down and scale bytes s1, s_up, s_down.  Rows outside every segment of
    a known expert are NaN."""
    a = row_values(*unpack_rows(rows, H))
    out = np.full((rows.shape[0], H), np.nan)
    value = {}
    for i, e in enumerate(seg_expert):
        lo, hi = int(seg_offset[i]), int(seg_offset[i + 1])
        if hi <= lo or not 0 <= e < len(experts):
            continue
        if e not in value:
            w = experts[e]
            value[e] = [weight_values(w["w" + n], w["s" + n]) if w.get("w" + n) is not None else None for n in ("1", "_up", "_down")]
        w1, w_up, w_down = value[e]
        h = activation(act, a[lo:hi] @ w1.T, a[lo:hi] @ w_up.T if act == ACT_SWIGLU else None)
        out[lo:hi] = row_values(*quantize_rows(h)) @ w_down.T
    return out
