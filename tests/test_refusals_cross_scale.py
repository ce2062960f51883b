"""Score scales that cross attention takes: 0, or what leaves a row's logarithm over the scale finite in 32 bits."""

import os

import pytest

from tests.test_refusals_layer import INVALID, LIB, _call, _cross, _cross_grad, _refused

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libravel.so not built")


@pytest.mark.parametrize("scale", [2.0 ** -101, 1e-38, 1e-45, -0.25, float("inf")])
def test_scales_out_of_range(scale):
    _refused(_call("ravel_cross_attention", _cross(scale=scale)), INVALID)
    _refused(_call("ravel_cross_attention_grad", _cross(scale=scale), _cross_grad()), INVALID)


@pytest.mark.parametrize("scale", [0.0, -0.0, 2.0 ** -100, 1e-20, 2.0 ** 100])
def test_scales_in_range(scale):
    assert _call("ravel_cross_attention", _cross(scale=scale, rows=0)) == 0
    assert _call("ravel_cross_attention_grad", _cross(scale=scale), _cross_grad(dq=None, dk=None, dv=None)) == 0
