"""What surrounds a block, rows in 8-bit integers and the layer of few tokens in fp64 (numpy), from the definitions in include/aurora_moe.h."""
from __future__ import annotations

import math

import numpy as np

from . import moe_layer

LEAST_SCALE = math.ldexp(1.0, -126)


def combine(ret, slot_to_row, topk_w, shared):
    """[rows,H], [T,k] (-1: dropped), [T,k], [T,H] or None -> [T,H], not rounded."""
    T, k = topk_w.shape
    y = np.zeros((T, ret.shape[1]))
    for t in range(T):
        for j in range(k):
            if slot_to_row[t, j] >= 0:
                y[t] += float(topk_w[t, j]) * np.asarray(ret[slot_to_row[t, j]], np.float64)
    return y if shared is None else y + np.asarray(shared, np.float64)


def rms_factor(v, eps):
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        return 1.0 / np.sqrt(np.mean(np.square(v), axis=1, keepdims=True) + float(np.float32(eps)))


def residual_sum(y, residual, gamma_post, gate, gate_tokens, scale, norm_post, eps):
    """r before it is rounded to the rows' type."""
    u = np.asarray(y, np.float64)
    if norm_post:
        u = u * rms_factor(u, eps)
        if gamma_post is not None:
            u = u * gamma_post
    if gate is not None:
        u = u * np.asarray(gate, np.float64)[np.arange(len(u)) // gate_tokens]
    u = u * float(np.float32(scale))
    return u if residual is None else u + residual


def normed(r, gamma_pre, eps):
    """v of the rounded r."""
    r = np.asarray(r, np.float64)
    v = r * rms_factor(r, eps)
    return v if gamma_pre is None else v * gamma_pre


def integer_scale(v):
    """[n,K] -> [n], NaN for a row that holds an infinity or a NaN"""
    with np.errstate(over="ignore", invalid="ignore"):
        s = (np.max(np.abs(v), axis=1) / 127.0).astype(np.float32).astype(np.float64)
    return np.where(np.isfinite(s), np.maximum(s, LEAST_SCALE), np.nan)


def integer_rows(v):
    """[n,K] -> whole numbers [n,K] (int8), scales [n] (fp32)"""
    s = integer_scale(v)
    fine = np.isfinite(s)
    q = np.zeros(v.shape)
    q[fine] = np.rint(v[fine] / s[fine, None])
    return q.astype(np.int8), s.astype(np.float32)


def int8_row_bytes(H):
    return -(-(H + 4) // 128) * 128


def pack_integer_rows(q, s):
    out = np.zeros((q.shape[0], int8_row_bytes(q.shape[1])), np.uint8)
    out[:, :q.shape[1]] = q.view(np.uint8)
    out[:, q.shape[1]:q.shape[1] + 4] = np.ascontiguousarray(s, np.float32).view(np.uint8).reshape(-1, 4)
    return out


def activation(act, a, up):
    if act == 1:
        return moe_layer._gelu_tanh(a)
    return moe_layer._silu(a) * (up if act == 2 else 1.0)


def round_bf16(v):
    """Nearest bf16 number, ties to even."""
    m, e = np.frexp(np.asarray(v, np.float64))
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def expert_ffn_int8(q, s, w, act):
    """Rows q [n,H], scales s [n] through one expert (int8 w1, w_up, w_down with fp32 scales s1, s_up, s_down per output channel)."""
    f = lambda a: np.asarray(a, np.float64)  # noqa: E731
    a = f(q) @ f(w["w1"]).T * f(w["s1"]) * f(s)[:, None]
    up = f(q) @ f(w["w_up"]).T * f(w["s_up"]) * f(s)[:, None] if act == 2 else None
    hq, hs = integer_rows(round_bf16(activation(act, a, up)))
    return f(hq) @ f(w["w_down"]).T * f(w["s_down"]) * f(hs)[:, None]


def layer_few(x, idx, topk_w, experts, local, act, shared=None):
    """y [T,H], not rounded: the experts that this GPU holds (local[e], -1: another one does), and the shared one."""
    x = np.asarray(x, np.float64)

    def expert(w, rows):
        f = lambda a: np.asarray(a, np.float64)  # noqa: E731
        up = rows @ f(w["w_up"]).T if act == 2 else None
        return activation(act, rows @ f(w["w1"]).T, up) @ f(w["w_down"]).T
    y = np.zeros_like(x) if shared is None else expert(shared, x)
    for t in range(x.shape[0]):
        for j in range(idx.shape[1]):
            e = int(idx[t, j])
            if 0 <= e < len(local) and local[e] >= 0:
                y[t] += float(topk_w[t, j]) * expert(experts[local[e]], x[t:t + 1])[0]
    return y
