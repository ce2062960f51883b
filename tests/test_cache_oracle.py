"""The cache oracle's own pins: codes against torch's e4m3 conversion, scales and eviction on cases written out by hand."""

import numpy as np
import torch

from tests import cache_oracle as co


def test_codes_are_torchs_e4m3():
    assert np.array_equal(co.DECODE, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(),
                          equal_nan=True)
    r = np.random.default_rng(1)
    x = np.concatenate([r.standard_normal(20000).astype(np.float32) * 2.0 ** r.integers(-14, 7, 20000), co.POSITIVE,
                        (co.POSITIVE[1:] + co.POSITIVE[:-1]) / 2, [-0.0, 0.0]]).astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(co.encode(x), want)
    assert co.DECODE[co.encode(np.inf)] == 448 and co.DECODE[co.encode(-np.inf)] == -448
    assert np.isnan(co.DECODE[co.encode(np.nan)])


def test_scales():
    for x, s in ((448.0, 1.0), (448.1, 2.0), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8), (1.7500001, 2.0 ** -7), (0.0, 2.0 ** -100),
                 (3e38, 2.0 ** 120), (1e-38, 2.0 ** -100)):
        assert co.scale_for([0.0, -x, np.nan, np.inf]) == s, x


def test_append_keeps_a_blocks_larger_scale_and_raises_a_smaller_one():
    c = co.new_cache(1, 1, 32, 32, 16)
    one = np.ones((1, 1, 1, 32), np.float32)
    co.append(c, 448 * one, one, pos=[0])
    co.append(c, one, 900 * one)
    assert c["ks"][0, 0, 0] == 1 and c["vs"][0, 0, 0] == 4 and c["len"][0] == 2
    assert np.all(co.DECODE[c["k"][0, 0, :2, 0]] == [448, 1])  # codes in units of the scale
    assert np.all(co.DECODE[c["v"][0, 0, :2, 0]] == [0.25, 224])  # 900 / 4 = 225, halfway to 240: nearest is 224


def test_eviction_fills_holes_in_order():
    c = co.new_cache(1, 1, 16, 32, 16)
    c["len"][0] = 8
    c["w"][0, 0, :8] = [0, 5, 1, 5, 9, 5, np.nan, 7]
    kept = co.evict(co.copy(c), 4)
    assert kept.tolist() == [[[4, 1, 7, 3]]]  # 9, 7, then the 5s of index 1 and 3
    kept = co.evict(c, 4, first=1)
    assert kept.tolist() == [[[0, 1, 4, 7]]]
    assert c["w"][0, 0, :4].tolist() == [0, 5, 9, 7] and c["len"][0] == 4
