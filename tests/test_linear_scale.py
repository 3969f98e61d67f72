"""A scale whose reciprocal passes f32 is refused where the gradients need it."""
import ctypes

import pytest

import paper_2606_25041_amd as ws
from tests import test_linear_abi as abi


@pytest.mark.parametrize("scale", (1e-39, 2.0 ** -149))
def test_gradients_of_a_tiny_scale(scale):
    lib = ws.library()
    assert ctypes.c_float(scale).value > 0
    assert abi.bwd(lib, scale=scale, ds=abi.FAKE) == abi.UNSUPPORTED
