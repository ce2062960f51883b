"""Accumulated weights, row by row: a row that is left out, counted twice or given another's sum shows up.

A weight is a sum over rows of p = exp(score - log sum): the score and the sum are off by the bound d of
test_gpu_cache.py with the largest size of the call's own inputs, the sum of `terms` numbers by (terms + 16) u, and the
logarithm's and the exponential's own rounding and that of their arguments (of a few tens at most) by 2^-18.
"""

import numpy as np
import pytest

from tests import cache_oracle as co
from tests.harness import have_gpu
from tests.test_gpu_cache import ATTEND, U, _bf16, _dev, _draw_cache, _ints, _tokens, _upload

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


def _track(g, c, q, ks, vs, dtype, seq):
    """One tracked call on both sides; (GPU's weights, the oracle's added ones, bound)."""
    import torch
    hd, before = q.shape[3], c["w"].astype(np.float64)
    dq = _dev(q, dtype)
    out = torch.empty_like(dq)
    own = [None if x is None else _dev(x, dtype) for x in (ks, vs)]
    g.attention(dq, out, *own, seq=_ints(seq), track=True)
    _, _, size = co.attention(c, q, ks, vs, seq=seq, track=True)
    added = c["w"] - before
    terms = 2 * q.shape[1] * q.shape[2] // c["k"].shape[1]
    rel = 2 * 2 * (hd + 6) * U * size.max() + 2.0 ** -18 + (terms + c["k"].shape[2] + 16) * U
    assert rel < 0.01  # of a key's weight: a row among a hundred shows
    torch.cuda.synchronize()
    return g.weight.cpu().numpy().astype(np.float64), added, rel * added + 2 * U * c["w"] + 1e-30


@pytest.mark.parametrize("hd,nq,nkv,block,cap,lens,rows,n_self,dtype",
                         ATTEND[:1] + ATTEND[2:9:2] + ATTEND[9:16] + ATTEND[18:30:2])
def test_against_the_inputs_own_size(hd, nq, nkv, block, cap, lens, rows, n_self, dtype):
    r = np.random.default_rng(hd + cap + rows + 4)
    c = _draw_cache(r, 4, nkv, cap, hd, block, lens + [cap])
    g = _upload(c)
    q = _tokens(r, 6, rows, nq, hd, dtype=dtype)
    ks, vs = (_tokens(r, 6, n_self, nkv, hd, dtype=dtype) if n_self else None for _ in range(2))
    got, _, lim = _track(g, c, q, ks, vs, dtype, [3, 0, 1, 3, 2, -1])
    assert (np.abs(got - c["w"]) <= lim).all()


@pytest.mark.parametrize("hd,nq,nkv,cap,rows,batch,dtype", [
    (256, 8, 1, 816, 50, 2, "bf16"),    # four waves share 64 keys
    (256, 8, 1, 700, 41, 1, "bf16"),    # rows that do not fill 32
    (128, 16, 4, 1100, 100, 2, "bf16"),
    (128, 16, 4, 500, 33, 1, "bf16"),
    (128, 16, 16, 4200, 7, 4, "bf16"),  # one wave to 64 keys
    (256, 8, 2, 300, 8, 2, "bf16"),     # few rows
    (256, 8, 1, 300, 25, 2, "f32"),
    (128, 6, 2, 400, 21, 1, "f32"),
])
def test_every_row_on_a_key_of_its_own(hd, nq, nkv, cap, rows, batch, dtype):
    """Row i of a KV head looks along key i's direction: that key's weight is this row's, nearly 1.  Two batch rows of one
    sequence count twice."""
    r = np.random.default_rng(hd + cap + rows + 5)
    c = _draw_cache(r, batch, nkv, cap, hd, 64, [cap] * batch)
    c["w"][:] = 0
    G = nq // nkv
    R = G * rows
    assert R <= cap
    seq = list(range(batch)) + [0]
    q = np.zeros((batch + 1, rows, nq, hd), np.float32)
    picks = {}
    for b, s in enumerate(seq):
        for h in range(nkv):
            k, _ = co.values(c, s, h, cap)
            if (s, h) not in picks:
                picks[s, h] = r.permutation(cap)[:R]
            k = k[picks[s, h]]
            x = 30.0 * np.sqrt(hd) * k / (k ** 2).sum(-1, keepdims=True)
            # row h' * rows + i of the KV head is query head h' at row i
            q[b, :, h * G:(h + 1) * G] = x.reshape(G, rows, hd).transpose(1, 0, 2)
    q = _bf16(q) if dtype == "bf16" else q
    g = _upload(c)
    got, added, lim = _track(g, c, q, None, None, dtype, seq)
    for (s, h), at in picks.items():  # the oracle alone: these are the inputs that tell rows apart
        own = added[s, h, at]
        assert np.median(own) > 0.9 * (2 if s == 0 else 1), (s, h, np.median(own))
    assert lim.max() < 0.05
    assert (np.abs(got - c["w"]) <= lim).all()
