"""Calls of many batch rows over few sequences, broadcast inputs, and destinations without weights."""

import numpy as np
import pytest

from tests import cache_oracle as co
from tests.harness import have_gpu
from tests.test_gpu_cache import U, _bound, _dev, _draw_cache, _ints, _same, _tokens, _upload

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("hd,nq,nkv,cap,rows,dtype", [(64, 8, 2, 200, 1, "bf16"), (128, 8, 2, 150, 20, "bf16"),
                                                       (32, 4, 1, 90, 3, "f32"), (256, 8, 1, 130, 50, "bf16")])
def test_many_rows_of_few_sequences(hd, nq, nkv, cap, rows, dtype):
    """150 batch rows over 7 sequences, named up to 140 rows apart: append and eviction take the first row of each, every
    row's weights count."""
    import torch
    r = np.random.default_rng(hd + cap)
    c = _draw_cache(r, 7, nkv, cap, hd, 16, [cap, 0, 33, cap // 2, 5, 16, cap - 1])
    g = _upload(c)
    B = 150
    seq = r.integers(-1, 5, B)  # 5 and 6 are named late and once
    seq[140], seq[149], seq[3] = 6, 5, 9
    k, v = _tokens(r, B, 3, nkv, hd, dtype=dtype), _tokens(r, B, 3, nkv, hd, dtype=dtype)
    g.append(_dev(k, dtype), _dev(v, dtype), seq=_ints(seq))
    co.append(c, k, v, seq=seq)
    _same(g, c)
    q, ks, vs = (_tokens(r, B, rows, h, hd, dtype=dtype) for h in (nq, nkv, nkv))
    dq, out = _dev(q, dtype), None
    out = torch.empty_like(dq)
    before = c["w"].astype(np.float64)
    g.attention(dq, out, _dev(ks, dtype), _dev(vs, dtype), seq=_ints(seq), track=True)
    want, absv, size = co.attention(c, q, ks, vs, seq=seq, track=True)
    got = out.float().cpu().numpy()
    assert (np.abs(got - want) <= _bound(dtype, hd, cap + rows, want, absv, size)).all()
    added = c["w"] - before
    terms = B * rows * nq // nkv
    # as in test_gpu_cache_weights.py, with a rounding more for every batch row added in turn
    rel = 2 * 2 * (hd + 6) * U * size.max() + 2.0 ** -18 + (terms + cap + 16 + B) * U
    assert (np.abs(g.weight.cpu().numpy() - c["w"]) <= rel * added + 2 * U * c["w"]).all()
    c["w"] = g.weight.cpu().numpy()
    kept = g.evict(20, first=1, seq=_ints(seq))
    assert np.array_equal(kept.cpu().numpy(), co.evict(c, 20, 1, seq=seq))
    _same(g, c)


def test_one_source_into_several_destinations_without_weights():
    r = np.random.default_rng(50)
    c = _draw_cache(r, 3, 2, 100, 64, 32, [100, 40, 7])
    d = co.new_cache(5, 2, 30, 64, 32, seed=2)
    gs, gd = _upload(c), _upload(d, weight=False)
    seq, into_seq = [0, 1, 0, 2, 0, 1], [4, 1, 0, 2, 4, -1]
    kept = gs.evict(25, first=3, seq=_ints(seq), into=gd, into_seq=_ints(into_seq))
    assert np.array_equal(kept.cpu().numpy(), co.evict(c, 25, 3, seq=seq, into=d, into_seq=into_seq))
    _same(gd, d, weight=False)
    _same(gs, c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_broadcast_inputs(dtype):
    """One token stored for every sequence, one row and one set of own tokens asked of every sequence: strides of 0."""
    import torch
    r = np.random.default_rng(51)
    nq, nkv, hd, B = 6, 2, 128, 4
    c = _draw_cache(r, B, nkv, 70, hd, 16, [70, 0, 13, 69])
    g = _upload(c)
    k, v = _tokens(r, 1, 1, 1, hd, dtype=dtype), _tokens(r, 1, 1, 1, hd, dtype=dtype)
    wide = lambda x, *s: np.broadcast_to(x, s + (hd,))  # noqa: E731
    g.append(_dev(k, dtype).expand(B, 2, nkv, hd), _dev(v, dtype).expand(B, 2, nkv, hd))
    co.append(c, wide(k, B, 2, nkv), wide(v, B, 2, nkv))
    _same(g, c)
    q = _tokens(r, 1, 1, nq, hd, dtype=dtype)
    dq = _dev(q, dtype).expand(B, 40, nq, hd)
    out = torch.empty((B, 40, nq, hd), dtype=dq.dtype, device="cuda")
    g.attention(dq, out, _dev(k, dtype).expand(B, 5, nkv, hd), _dev(v, dtype).expand(B, 5, nkv, hd))
    want, absv, size = co.attention(c, np.broadcast_to(q, (B, 40, nq, hd)), wide(k, B, 5, nkv), wide(v, B, 5, nkv))
    assert (np.abs(out.float().cpu().numpy() - want) <= _bound(dtype, hd, 75, want, absv, size)).all()


def test_calls_without_rows_and_tokens():
    """An empty batch and no own tokens given as empty tensors do nothing more than that."""
    import torch
    r = np.random.default_rng(52)
    c = _draw_cache(r, 2, 2, 50, 64, 16, [50, 20])
    g = _upload(c)
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    g.append(e(0, 3, 2, 64), e(0, 3, 2, 64), seq=none)
    g.append(e(2, 0, 2, 64), e(2, 0, 2, 64))
    g.attention(e(0, 3, 4, 64), e(0, 3, 4, 64), seq=none, track=True)
    assert g.evict(5, seq=none).shape == (0, 2, 5)
    _same(g, c)
    q = _tokens(r, 2, 3, 4, 64, dtype="bf16")
    outs = [torch.empty((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    g.attention(_dev(q, "bf16"), outs[0], e(2, 0, 2, 64), e(2, 0, 2, 64))
    g.attention(_dev(q, "bf16"), outs[1])
    assert torch.equal(*outs)
