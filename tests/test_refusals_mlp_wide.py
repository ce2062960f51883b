"""Gate and up values in 32 bits (RAVEL_GATE_F32): what the checks make of their rows."""

import os

import pytest

from tests.test_refusals_layer import INVALID, LIB, SHAPE, _call, _mlp, _mlp_grad, _refused, _ravel

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libravel.so not built")


def test_the_flag_is_the_headers():
    text = open(os.path.join(os.path.dirname(os.path.dirname(LIB)), "include", "ravel.h")).read()
    assert f"RAVEL_GATE_F32 = {_ravel().GATE_F32}" in text


@pytest.mark.parametrize("kw,status", [
    (dict(act=2 | 256), INVALID), (dict(act=512), INVALID), (dict(act=-1), INVALID), (dict(act=256, gate_stride=120), SHAPE),
    (dict(act=257, gate_stride=130), SHAPE), (dict(act=257, gate=None), INVALID), (dict(act=256, gate=(1 << 20) + 8), INVALID),
    (dict(act=256, gate_stride=1 << 21), SHAPE)])
def test_refused(kw, status):
    _refused(_call("ravel_gated_mlp", _mlp(**kw)), status)


def test_strides_of_16_bytes():
    """4 numbers of 32 bits where 8 of bf16 are needed; found in range (nothing is wanted, so nothing is launched)."""
    none = dict(dx=None, dwg=None, dwu=None)
    assert _call("ravel_gated_mlp_grad", _mlp(act=256, gate_stride=132), _mlp_grad(**none)) == 0
    _refused(_call("ravel_gated_mlp_grad", _mlp(act=0, gate_stride=132), _mlp_grad(**none)), SHAPE)
    assert _call("ravel_gated_mlp_grad", _mlp(act=257, dtype=0, gate_stride=132), _mlp_grad(weight_dtype=0, **none)) == 0
