"""Cross attention with its gradients at the smallest and at large score scales."""

import pytest

from tests import layer_oracle as lo
from tests.harness import have_gpu
from tests.test_gpu_cross_attention import _case, _compare, _run

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [2.0 ** -100, 1e-20])
@pytest.mark.parametrize("R,K", [(20, 50), (70, 300), (9, 16)])
def test_scales_that_leave_the_mean(dtype, scale, R, K):
    c = _case(dtype, (8, 2, 64), 2, R, K, None, [K, K - 3], scale=scale)
    _, _, got = _run(c)
    _compare(c, got)
    assert bool(got["dv"].any()) and bool(got["dk"].any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small_queries_under_the_largest_scale(dtype):
    c = _case(dtype, (8, 2, 64), 2, 20, 50, None, [50, 47], scale=2.0 ** 100)
    c["q"] = lo.held(c["q"] * 2.0 ** -103, dtype)
    _, _, got = _run(c)
    _compare(c, got)
