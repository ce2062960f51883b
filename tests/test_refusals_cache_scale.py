"""A score scale whose product with log2 e is infinite would turn scores of 0 into NaN: refused from 2^100 on."""

import pytest

from tests.test_refusals_cache import INVALID, _attend, _cache, _lib, _query
from tests.test_refusals_cache import pytestmark  # noqa: F401


@pytest.mark.parametrize("scale", [3e38, 2.0 ** 127, 2.0 ** 101])
def test_large_scales(scale):
    q = dict(out=1 << 30, workspace=1 << 32)
    assert _attend(_cache(), _query(scale=scale, **q)) == INVALID
    assert b"scale" in _lib().ravel_last_error()


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -149, 1.0, 2.0 ** 100])
def test_scales_in_range(scale):
    assert _attend(_cache(), _query(scale=scale, batch=0)) == 0
