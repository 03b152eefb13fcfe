"""What a bf16 layer for a few tokens rounds: its inner activations to 2^-17, y once.  Bounds in tests/few_checks.py."""
import numpy as np
import pytest
import torch

from tests import few_checks as K
from tests.test_gpu_layer_few import Layer

pytestmark = pytest.mark.gpu


# up to 8, 16, 32 and 64 tokens of an expert in a product, of the shared one and of the others; the last ones on their own, and the shared one on its own
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("T", [1, 8, 9, 16, 17, 32, 33, 64])
def test_rounded_once(T, act):
    H, F = (1024, 512) if T == 1 else (512, 384)
    for local, Fs in ((None, 128), (None, 0), ([-1] * 3, 256)):
        c = Layer(T, H, F, 3, 2, act=act, local=local, F_shared=Fs).check()
        K.assert_rounded_once(c.y.double().cpu().numpy(), c.want(c.idx.cpu().numpy(), c.w.cpu().numpy()))


def test_rounded_once_with_64_tokens_at_one_expert():
    c = Layer(64, 640, 256, 40, 3).device()                                  # and a few at each of many
    rng = np.random.default_rng(2)
    others = np.stack([rng.permutation(39)[:2] for _ in range(64)]) + 1
    idx, w = np.insert(others, 1, 0, axis=1).astype(np.int32), rng.uniform(0.2, 0.5, (64, 3)).astype(np.float32)
    c.idx.copy_(torch.from_numpy(idx))
    c.w.copy_(torch.from_numpy(w))
    c.bind(routed=True)()
    K.assert_rounded_once(c.y.double().cpu().numpy(), c.want(idx, w))
