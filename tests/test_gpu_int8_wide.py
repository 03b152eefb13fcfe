"""The integer FFN on few rows of layers wider than 32768, bit for bit as in tests/test_gpu_int8.py."""
import numpy as np
import pytest

from tests.test_gpu_int8 import GELU, SILU, SWIGLU, check_bits
from tests.test_int8_plans import plan_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", [SILU, GELU, SWIGLU])
@pytest.mark.parametrize("R,Hn,F,n_local,mt", [(1, 128, 33024, 1, 1), (20, 256, 32896, 1, 2), (60, 128, 130944, 1, 4), (5, 33024, 128, 1, 1), (130, 32896, 256, 2, 4), (90, 256, 33024, 4, 2)])
def test_streamed(R, Hn, F, n_local, mt, act):
    plan = plan_of(R, n_local, n_local, Hn, F, act)
    assert plan[0] == mt, plan
    check_bits(np.random.default_rng([R, Hn, F]), R, Hn, F, act, [R * i // n_local for i in range(n_local + 1)], list(range(n_local)), n_local)
