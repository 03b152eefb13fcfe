"""Bounds that tell a y which was rounded once from one whose inner activations were rounded to bf16 before.

With the inner activations kept to 2^-17 (half a step of the second bf16 number) y, before its rounding, is off by at most 2^-17 / sqrt(3) = 4.4e-6 of its norm, as the
errors of a row's activations are independent; sums in fp32, the activation's exponential and reciprocal (some 1e-6 of an activation) and the choices' weights (2^-24) add less.  So

- an element is another bf16 number than the oracle's only if the middle of two lies in between: error / step in probability, where a step is 2^-7.5 of an element: 3.5e-6
  (the mean of such an error) * 181 * the mean of norm / |element| (some 5.5 for normal elements, a thousandth of the norm at least) = 0.0035.  FLIPS is six times that.
- the squares of such errors are nothing beside those of y's own rounding, 2^-8 / sqrt(3) and less: RMS leaves 2 %.

An activation rounded once to bf16 is off by up to 2^-8, and both fail: the error is then that of y's own rounding again (sqrt(2) times it together), and elements turn into other ones
by the third."""
import numpy as np

from oracle import block_layer as B

FLIPS, RMS = 0.02, 1.02


def against(got, want):
    """Share of elements that are not the nearest bf16 number of the oracle's 64-bit value, and the error in units of that number's."""
    got, nearest = np.asarray(got, np.float64), B.round_bf16(want)
    rms = lambda v: np.sqrt(np.mean(np.square(v)))  # noqa: E731
    return np.mean(got != nearest), rms(got - want) / rms(nearest - want)


def assert_rounded_once(got, want):
    flips, rms = against(got, want)
    assert flips <= FLIPS and rms <= RMS, (flips, rms)


def layer(x, idx, topk_w, experts, local, act, shared, hold):
    """B.layer_few with the inner activations held as `hold` leaves them."""
    x = np.asarray(x, np.float64)

    def expert(w, rows):
        up = rows @ w["w_up"].T if act == 2 else None
        return hold(B.activation(act, rows @ w["w1"].T, up)) @ w["w_down"].T
    y = np.zeros_like(x) if shared is None else expert(shared, x)
    for t in range(x.shape[0]):
        for j in range(idx.shape[1]):
            if local[idx[t, j]] >= 0:
                y[t] += float(topk_w[t, j]) * expert(experts[local[idx[t, j]]], x[t:t + 1])[0]
    return y


def one(h):
    return B.round_bf16(h)


def two(h):
    hi = B.round_bf16(h)
    return hi + B.round_bf16(h - hi)
