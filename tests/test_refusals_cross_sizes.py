"""What the gradients of cross attention ask for where there are many heads and few rows: no more than the rows that there are
need.  Answered on the host, before anything is launched."""

import ctypes
import os

import pytest

from tests.test_refusals_layer import LIB, SHAPE, _cross, _cross_grad, _ravel

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libravel.so not built")


def _workspace(cross, grad):
    lib, n = _ravel().load_library(), ctypes.c_int64(-1)
    status = lib.ravel_cross_attention_grad_workspace(ctypes.byref(cross), ctypes.byref(grad), ctypes.byref(n))
    return status, n.value


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("head_dim", [32, 64, 128, 256])
@pytest.mark.parametrize("heads,rows", [((1, 1), 1), ((8, 1), 1), ((2, 2), 17), ((4, 1), 8)])
def test_statistics_of_the_rows_that_there_are(dtype, head_dim, heads, rows):
    """Two numbers of 32 bits a row, in tiles of at most 64 rows of a KV head; no sums of ranges where the heads fill the chip."""
    nq, nkv = heads
    status, n = _workspace(_cross(dtype=dtype, batch=20000, n_q_heads=nq, n_kv_heads=nkv, head_dim=head_dim, rows=rows, keys=40), _cross_grad())
    tile = 64 if head_dim * (4 if dtype == 0 else 2) >= 512 else 32
    assert status == 0
    assert 0 < n <= 20000 * nkv * -(-rows * nq // nkv // tile) * tile * 8 + 255


def test_sizes_that_a_launch_does_not_hold():
    """Blocks of 256 threads, below 2^32 of them: (batch rows times KV heads) 2^21 with one tile of rows and three of keys, or as
    many as there can be with dq alone, are in range; a second tile for as many is not."""
    many = dict(n_q_heads=64, n_kv_heads=64, head_dim=32, rows=1, keys=33)
    assert _workspace(_cross(batch=32768, **many), _cross_grad()) == (0, 32768 * 64 * 16 * 8)
    most = dict(n_q_heads=256, n_kv_heads=256, head_dim=32, keys=64)
    alone = _cross_grad(dk=None, dv=None)
    assert _workspace(_cross(batch=65535, rows=1, **most), alone) == (0, 0)
    assert _workspace(_cross(batch=65535, rows=17, **most), alone)[0] == SHAPE
    assert _workspace(_cross(batch=65535, rows=1, **most), _cross_grad())[0] == SHAPE  # four tiles of keys
    assert _workspace(_cross(batch=16383, rows=1, **most), _cross_grad())[0] == 0
