"""Caps and scales far from each other and from 1: the polynomials' coefficients have powers of their ratio in them."""
import pytest

from attention_reference import THETA, Scene
from paper_2508_08895_b200 import binding as B
from test_gpu_scores import SMALL, TC, bits

pytestmark = pytest.mark.gpu

STEP = [(90, [(20, 1), (3, 2)], 0), (5, [(0, 4)], 0)]


# queries so large that scores reach half of the cap, or a few units where that is more
@pytest.mark.parametrize("sm_scale,cap,q_scale", [(9e10, 1e6, 2e-12), (9e10, 50.0, 2e-11), (1e-7, 50.0, 4e6), (1e-12, 3.0, 4e10), (0.125, 1e-7, 1e-6), (1e5, 2.0, 1e-6),
                                                  (3e-4, 20.0, 3e3), (1.0, 1e5, 0.3)])
@pytest.mark.parametrize("shape", [TC, SMALL[0], SMALL[1]], ids=str)
def test_scales(shape, sm_scale, cap, q_scale):
    s = Scene(*shape, STEP, cap=cap, q_scale=q_scale)
    s.scale = sm_scale
    s.shape = B.make_shape(*shape[3], shape[1], shape[2], shape[0], THETA, sm_scale)
    s.step()
    s.check(**bits(shape))
