"""Attention over the 8-bit cache with a scale of 0, or so small that every score rounds to 0: the mean of the values.

Every probability is the same, and what a stage of keys masks stays masked.  Bounds are those of test_gpu_cache.py (the
scores' part of them is 0 here); a key's weight is a sum of R = rows * heads equal terms and so is off by (R + n + 16) u
of it, and by 2^-21 for the logarithm and the exponential of each.
"""

import numpy as np
import pytest

from tests.harness import have_gpu
from tests.test_gpu_cache import U, _attend, _draw_cache, _upload

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]

SHAPES = [
    # hd, nq, nkv, block, cap, lengths, rows, n_self, dtype: every head dim with many rows, then few, then 32 bits
    (256, 8, 1, 64, 7800, [7800, 0, 1999], 50, 50, "bf16"),
    (256, 8, 1, 16, 3001, [2977, 65, 64], 41, 0, "bf16"),
    (128, 16, 4, 128, 1100, [1100, 129, 1000], 100, 130, "bf16"),
    (64, 12, 3, 16, 2601, [2601, 2599, 5], 100, 7, "bf16"),
    (32, 4, 4, 32, 6300, [6300, 1, 1025], 128, 8, "bf16"),
    (128, 6, 2, 32, 129, [128, 129, 2], 17, 5, "bf16"),
    (64, 12, 3, 64, 301, [301, 299, 1], 85, 85, "bf16"),
    (64, 8, 8, 32, 257, [257, 0, 100], 16, 16, "f32"),
]


@pytest.mark.parametrize("scale", [0.0, 2.0 ** -149])
@pytest.mark.parametrize("hd,nq,nkv,block,cap,lens,rows,n_self,dtype", SHAPES)
def test_scale_zero(hd, nq, nkv, block, cap, lens, rows, n_self, dtype, scale):
    r = np.random.default_rng(hd + cap + rows + 2)
    c = _draw_cache(r, 4, nkv, cap, hd, block, lens + [0])
    before = c["w"].astype(np.float64)
    g = _upload(c)
    seq = [2, 0, -1, 1, 0, 3]
    _attend(g, c, r, dtype, nq, rows, n_self, 6, seq=seq, track=True, scale=scale)
    got = g.weight.cpu().numpy().astype(np.float64)
    added = c["w"] - before
    terms = 2 * rows * nq // nkv
    lim = (2.0 ** -21 + (terms + cap + n_self + 16) * U) * added + 2 * U * c["w"]
    assert (np.abs(got - c["w"]) <= lim).all()
    for s in range(4):
        assert np.array_equal(got[s, :, c["len"][s]:], before[s, :, c["len"][s]:])
