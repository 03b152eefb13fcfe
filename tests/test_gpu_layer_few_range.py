"""The layer for a few tokens with inner activations at the end of fp32's range, on the GPU."""
import numpy as np
import pytest
import torch

from tests import harness as H
from tests.test_gpu_layer_few import Layer

pytestmark = pytest.mark.gpu

MOST = 1.9921875 * 2.0 ** 127                                                # of bf16; fp32 has 2^127 (2 - 2^-23)
TOP = MOST + 1.5 * 2.0 ** 119                                                # rounds to a bf16 infinity


@pytest.mark.parametrize("T", [3, 13, 40])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("of_shared", [False, True])
def test_an_activation_between_the_largest_of_bf16_and_of_fp32(T, act, of_shared):
    """One inner activation of token 1 is TOP, finite, and weights of 2^-120 bring it back to 256 or so; token 2's is an infinity, which y has to be too.  bf16's largest number
    holds TOP to 2^-8 and a second one the rest to 2^-17, so that y is the oracle's within the bound of all these tests."""
    c = Layer(T, 512, 384, 3, 2, act=act, F_shared=384)
    weights = c.shared if of_shared else c.experts[1]
    for name in ("w1", "w_up"):
        if c.shared[name] is not None:
            for e in c.experts + [c.shared]:
                e[name][:, :3] = 0
    c.x[:, :3] = 0
    # every factor a bf16 number, TOP = 2^64 (MOST / 2^64) + 2^60 (1.5 2^59) in the sums; SwiGLU: that over 2^40, times an up of -2^40
    shift = 2.0 ** -40 if act == 2 else 1.0
    c.x[1, :3], c.x[2, :3] = [2.0 ** 64, 2.0 ** 60, 1.0], [2.0 ** 65, 0.0, 1.0]
    weights["w1"][7, :] = 0
    weights["w1"][7, :2] = [MOST / 2.0 ** 64 * shift, 1.5 * 2.0 ** 59 * shift]
    if act == 2:
        weights["w_up"][7, :] = 0
        weights["w_up"][7, 2] = -2.0 ** 40
    sign = -1.0 if act == 2 else 1.0
    weights["w_down"][:, 7] = 2.0 ** -120
    c.device()
    c.idx.copy_(torch.tensor([[1, 0]] * T, dtype=torch.int32))
    c.w.copy_(torch.tensor([[0.75, 0.25]] * T))
    c.bind(routed=True)()
    y = c.y.double().cpu().numpy()
    with np.errstate(over="ignore"):
        want = c.want(c.idx.cpu().numpy(), c.w.cpu().numpy())
    far = 2.0 ** -120 * TOP * sign * (1.0 if of_shared else 0.75)
    assert np.all(np.abs(want[1] - far) < 40)                                # the large activation counts
    H.assert_close(y[1:2], want[1:2], "bf16")
    assert np.all(y[2] == sign * np.inf)
    rest = [t for t in range(T) if t not in (1, 2)]
    H.assert_close(y[rest], want[rest], "bf16")
