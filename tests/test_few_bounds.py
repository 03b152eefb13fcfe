"""That the bounds on the layer for a few tokens see what they are for, by the oracle."""
import numpy as np
import pytest

from oracle import block_layer as B
from tests import few_checks as K


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("T,H,F,Fs,routed", [(1, 1024, 512, 128, True), (9, 512, 384, 0, True), (33, 512, 384, 256, False)])
def test_rounding_the_inner_activations_once_shows(T, H, F, Fs, routed, act):
    rng = np.random.default_rng([T, act])
    g = lambda s, *n: B.round_bf16(s * rng.standard_normal(n))  # noqa: E731
    weights = lambda f: {"w1": g(H ** -0.5, f, H), "w_up": g(H ** -0.5, f, H), "w_down": g(f ** -0.5, H, f)}  # noqa: E731
    experts, shared = [weights(F) for _ in range(3)], weights(Fs) if Fs else None
    local = [0, 1, 2] if routed else [-1] * 3
    x, idx, w = g(1.0, T, H), np.stack([rng.permutation(3)[:2] for _ in range(T)]), rng.random((T, 2)).astype(np.float32)
    want = B.layer_few(x, idx, w, experts, local, act, shared)
    K.assert_rounded_once(B.round_bf16(K.layer(x, idx, w, experts, local, act, shared, K.two)), want)
    flips, rms = K.against(B.round_bf16(K.layer(x, idx, w, experts, local, act, shared, K.one)), want)
    assert flips > 5 * K.FLIPS and rms > 1.2
    if Fs and routed:                                                        # of the shared expert alone, or of the others alone
        rest = lambda hold: K.layer(x, idx, w, experts, local, act, None, hold)  # noqa: E731
        mine = lambda hold: K.layer(x, idx, w, experts, [-1] * 3, act, shared, hold)  # noqa: E731
        for y in (rest(K.one) + mine(K.two), rest(K.two) + mine(K.one)):
            flips, rms = K.against(B.round_bf16(y), want)
            assert flips > K.FLIPS and rms > K.RMS
