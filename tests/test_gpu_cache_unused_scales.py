"""Scales of blocks behind a sequence's last token are never part of a result: a caller may leave them uninitialised."""

import numpy as np
import pytest

from tests.harness import have_gpu
from tests.test_gpu_cache import ATTEND, _attend, _draw_cache, _same, _upload

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("hd,nq,nkv,block,cap,lens,rows,n_self,dtype", ATTEND[1:4] + ATTEND[9:10] + ATTEND[13:18] + ATTEND[22:29])
def test_unused_scales(hd, nq, nkv, block, cap, lens, rows, n_self, dtype, value):
    r = np.random.default_rng(hd + cap + rows + 3)
    # lengths that end a few tokens into a block, so that the stage that holds the last one has blocks without any
    short = max(cap // 3 // block * block + 1, 1)
    c = _draw_cache(r, 5, nkv, cap, hd, block, lens + [short, 0])
    for s in range(5):
        used = -(-int(c["len"][s]) // block)
        for x in ("k", "v"):
            c[x + "s"][s, :, used:] = value
            c[x][s, :, c["len"][s]:] = 0x7F
    g = _upload(c)
    _attend(g, c, r, dtype, nq, rows, n_self, 6, seq=[2, 0, 3, 1, -1, 4], track=True)
    c["w"] = g.weight.cpu().numpy()
    assert np.isfinite(c["w"]).all()
    _same(g, c)
