"""Strides up to what the cache's own limits allow: 2^24 tokens of any head count are a legal source."""

import pytest

from tests.harness import have_gpu
from tests.test_refusals_cache import SHAPE, _append, _attend, _cache, _query
from tests.test_refusals_cache import pytestmark as built


class TestOnTheHost:
    pytestmark = built

    @pytest.mark.parametrize("st", [(1 << 30, 512, 64), (1 << 36, 1 << 12, 64), (1 << 33, 1 << 33, 1 << 33)])
    def test_long_strides_are_taken(self, st):
        # a batch of no rows: every check runs, nothing is launched
        assert _append(_cache(), batch=0, k=None, v=None, st=st) == 0

    def test_offsets_past_64_bits_are_not(self):
        assert _append(_cache(), st=(1 << 62, 128, 64)) == SHAPE
        assert _append(_cache(), st=(512, 1 << 60, 64)) == SHAPE
        assert _attend(_cache(), _query(q_stride=(1024, 1 << 60, 64))) == SHAPE
        assert _attend(_cache(), _query(self_stride=(1 << 61, 128, 64))) == SHAPE


@pytest.mark.gpu
@pytest.mark.skipif(not have_gpu(), reason="needs a GPU")
def test_a_row_with_a_long_batch_stride():
    """One row of a tensor whose rows would lie 2^31 elements apart: append and attention take it as any other."""
    import torch
    from paper_2609_34170_amd import ravel
    g = torch.Generator("cuda").manual_seed(0)
    k, v = (torch.randn((1, 5, 2, 64), generator=g, device="cuda") for _ in range(2))
    q = torch.randn((1, 3, 4, 64), generator=g, device="cuda")
    far = lambda x: x.as_strided(x.shape, (1 << 31,) + x.stride()[1:])  # noqa: E731
    outs = []
    for wrap in (lambda x: x, far):
        c = ravel.Cache.empty(1, 2, 20, 64, block=16)
        c.append(wrap(k), wrap(v))
        out = torch.empty_like(q)
        c.attention(wrap(q), wrap(out), wrap(k), wrap(v))
        torch.cuda.synchronize()
        outs.append((c.k.view(torch.uint8), c.k_scale, c.length, out))
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    assert outs[0][2].tolist() == [5]
