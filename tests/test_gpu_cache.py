"""The 8-bit key/value cache on the GPU against its definition in numpy (tests/cache_oracle.py).

Codes, scales, lengths, indices and moved weights are equal.  Attention is held to a bound derived per output from
the roundings that the operator makes (u = 2^-24):

* a score is a sum of hd products exact in 32 bits (8-bit by 8-bit significands; 32-bit queries in three exact parts),
  so it is off by at most (hd + 4) u size, size = scale sum |q| |k|, and its exponent's rounding by 2 u |score| <= 2 u
  size; a probability by the factor exp of twice that (the row's maximum may be off too), and by 2^-22 for the
  exponential: d = 2 (hd + 6) u size + 2^-22;
* bf16 calls round a probability (2^-8) and the output (2^-8); 32-bit calls neither;
* sums over n keys add n u.

So |out - exact| <= (d + [2^-8] + (n + 16) u) sum p |v| + (2^-8 or u) |exact|, the denominator's error taken in by
counting d and the sums twice.
"""

import numpy as np
import pytest

from tests import cache_oracle as co
from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]
U = 2.0 ** -24


def _bf16(x):
    """float32 values rounded to bf16 (to nearest even), as float32."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    return ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def _dev(x, dtype="f32"):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _upload(c, weight=True):
    from paper_2609_34170_amd import ravel
    return ravel.Cache(_dev(c["k"]), _dev(c["v"]), _dev(c["ks"]), _dev(c["vs"]), _dev(c["len"]), c["block"],
                       weight=_dev(c["w"].astype(np.float32)) if weight else None)


def _ints(x):
    return None if x is None else _dev(np.asarray(x, np.int32))


def _same(g, c, weight=True):
    """The whole memory is equal: what a call does not write stays as it was."""
    import torch
    torch.cuda.synchronize()
    for name, t, want in (("k", g.k, c["k"]), ("v", g.v, c["v"]), ("ks", g.k_scale, c["ks"]), ("vs", g.v_scale, c["vs"]),
                          ("len", g.length, c["len"])) + ((("w", g.weight, c["w"]),) if weight else ()):
        got = t.view(torch.uint8).cpu().numpy() if name in "kv" else t.cpu().numpy()
        if name in "kv":  # NaN has two codes
            got, want = (np.where(x & 0x7F == 0x7F, 0x7F, x) for x in (got, want))
            assert np.array_equal(got, want), (name, np.argwhere(got != want)[:5])
        else:
            assert np.array_equal(got, want.astype(got.dtype), equal_nan=True), name


def _tokens(r, *shape, dtype="f32"):
    x = (r.standard_normal(shape) * np.exp(0.5 * r.standard_normal(shape[-1]))).astype(np.float32)
    return _bf16(x) if dtype == "bf16" else x


def _draw_cache(r, n_seq, nkv, cap, hd, block, lens):
    """Filled through the oracle's append up to lens, stale behind."""
    c = co.new_cache(n_seq, nkv, cap, hd, block, seed=int(r.integers(1 << 30)))
    n = max(max(lens), 1)
    co.append(c, _tokens(r, n_seq, n, nkv, hd), _tokens(r, n_seq, n, nkv, hd), pos=[0] * n_seq, count=lens)
    c["w"] = r.random(c["w"].shape, dtype=np.float32)
    return c


# ---------------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("hd,nkv,cap,block,dtype,n", [
    (32, 3, 50, 16, "bf16", 37), (64, 1, 129, 32, "f32", 129), (128, 2, 200, 64, "bf16", 1), (256, 1, 300, 128, "f32", 150),
    (256, 2, 257, 16, "bf16", 100), (64, 5, 31, 128, "f32", 31), (128, 1, 1, 64, "bf16", 1)])
def test_append(hd, nkv, cap, block, dtype, n):
    r = np.random.default_rng(hd + n)
    c = _draw_cache(r, 6, nkv, cap, hd, block, [0, cap, cap // 2, 1, cap // 3, cap])
    g = _upload(c)
    seq = [4, 0, 5, -1, 2, 6, 1]  # sequence 3 is not named, two rows name none
    pos = [min(cap, 17), 0, cap // 2, 0, cap, 0, cap + 1]  # the last is out of range
    count = [n, max(n - 3, 0), n, n, n, n, n]
    k, v = _tokens(r, 7, n, nkv, hd, dtype=dtype), _tokens(r, 7, n, nkv, hd, dtype=dtype) * np.float32(16)
    g.append(_dev(k, dtype), _dev(v, dtype), pos=_ints(pos), count=_ints(count), seq=_ints(seq))
    co.append(c, k, v, pos=pos, count=count, seq=seq)
    _same(g, c)


def test_append_at_the_lengths_token_by_token():
    """A decode loop without positions: scales grow inside a block, the capacity is a bound, lengths out of range are clamped."""
    r = np.random.default_rng(3)
    c = _draw_cache(r, 3, 2, 40, 64, 16, [0, 7, 38])
    c["len"][0] = -5
    g = _upload(c)
    for i in range(24):
        k = _tokens(r, 3, 1, 2, 64, dtype="bf16") * np.float32(2.0 ** (i % 7))
        v = _tokens(r, 3, 1, 2, 64, dtype="bf16") / np.float32(2.0 ** (i % 5))
        g.append(_dev(k, "bf16"), _dev(v, "bf16"), pos=g.length if i % 2 else None)
        co.append(c, k, v)
    assert c["len"].tolist() == [24, 31, 40]
    _same(g, c)


def test_append_extremes():
    """Zeros, values over and under every scale, infinities, NaN, halves between codes, a sequence named twice, n = 0."""
    r = np.random.default_rng(4)
    c = co.new_cache(4, 1, 64, 32, 16, seed=5)
    k = _tokens(r, 5, 16, 1, 32)
    v = k.copy()
    k[0] = 0.0
    k[1] = np.clip(k[1].astype(np.float64) * 1e38, -3e38, 3e38)
    k[1, 3, 0, 5], k[1, 4, 0, 6], k[1, 5, 0, 7] = np.inf, -np.inf, np.nan
    v[1] *= np.float32(1e-38)
    k[2] = np.resize(np.concatenate([(co.POSITIVE[1:] + co.POSITIVE[:-1]) / 2, -co.POSITIVE]), k[2].shape)
    v[2] = np.nan
    v[0, :, 0, 0] = np.inf
    g = _upload(c)
    seq = [0, 1, 3, 1, 2]
    g.append(_dev(k), _dev(v), pos=_ints([0] * 5), seq=_ints(seq))
    co.append(c, k, v, pos=[0] * 5, seq=seq)
    _same(g, c)
    # raise the scale over stored NaN, infinities and subnormal codes
    big = np.full((4, 3, 1, 32), 2.0 ** 30, np.float32)
    g.append(_dev(big), _dev(big), pos=_ints([15, 14, 9, 3]))
    co.append(c, big, big, pos=[15, 14, 9, 3])
    _same(g, c)
    g.append(_dev(big[:, :0]), _dev(big[:, :0]), pos=_ints([2, 2, 2, 2]))  # takes tokens back
    co.append(c, big[:, :0], big[:, :0], pos=[2] * 4)
    _same(g, c)
    assert c["len"].tolist() == [2] * 4


def test_append_strided_sources():
    """Keys and values inside a wider projection's rows, head by head or token by token."""
    import torch
    r = np.random.default_rng(6)
    for order in ((0, 1, 2, 3), (0, 2, 1, 3)):
        c = _draw_cache(r, 2, 2, 70, 128, 32, [70, 3])
        g = _upload(c, weight=False)
        x = _tokens(r, 2, 33, 2, 3 * 128, dtype="bf16")
        full = _dev(x.transpose(order), "bf16").permute(order)
        k, v = full[..., 128:256], full[..., 256:]
        assert not k.is_contiguous()
        g.append(k, v, pos=_ints([30, 5]))
        co.append(c, x[..., 128:256], x[..., 256:], pos=[30, 5])
        _same(g, c, weight=False)


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
def _bound(dtype, hd, keys, out, absv, size):
    d = 2 * (hd + 6) * U * size[..., None] + 2.0 ** -22
    rnd = 2.0 ** -8 if dtype == "bf16" else 0.0
    return 2 * (d + (keys + 16) * U) * absv + rnd * absv + (2.0 ** -8 if dtype == "bf16" else 2 * U) * np.abs(out) + 1e-30


def _attend(g, c, r, dtype, nq, rows, n_self, batch, seq=None, track=False, scale=None, packed=False):
    """One call on both sides, compared; returns the oracle's output."""
    import torch
    nkv, cap, hd = c["k"].shape[1:]
    q = _tokens(r, batch, rows, nq, hd, dtype=dtype)
    ks, vs = (_tokens(r, batch, n_self, nkv, hd, dtype=dtype) for _ in range(2))
    if packed and n_self == rows:  # one projection's rows, as a layer writes them
        x = _dev(np.concatenate([q, ks, vs], 2), dtype)
        dq, dk, dv = x[:, :, :nq], x[:, :, nq:nq + nkv], x[:, :, nq + nkv:]
    else:
        dq, dk, dv = _dev(q, dtype), _dev(ks, dtype), _dev(vs, dtype)
    out = torch.full((batch, nq, rows, hd), float("nan"), dtype=dq.dtype, device="cuda").permute(0, 2, 1, 3)
    none = n_self == 0
    g.attention(dq, out, None if none else dk, None if none else dv, seq=_ints(seq), track=track, scale=scale)
    want, absv, size = co.attention(c, q, None if none else ks, None if none else vs, seq=seq, scale=scale, track=track)
    torch.cuda.synchronize()
    got = out.float().cpu().numpy().astype(np.float64)
    lim = _bound(dtype, hd, cap + n_self, want, absv, size)
    bad = ~(np.abs(got - want) <= lim)
    assert not bad.any(), (np.argwhere(bad)[:3], np.abs(got - want)[bad][:3], lim[bad][:3])
    return want


ATTEND = [
    # hd, nq, nkv, block, cap, lengths, rows, n_self, dtype
    (256, 8, 1, 64, 816, [816, 0, 333], 50, 50, "bf16"),
    (256, 8, 1, 128, 70, [70, 1, 64], 1, 0, "bf16"),
    (128, 16, 4, 64, 700, [700, 31, 33], 100, 100, "bf16"),
    (128, 16, 4, 16, 2100, [2100, 0, 1999], 1, 1, "bf16"),
    (128, 6, 2, 32, 129, [128, 129, 2], 17, 5, "bf16"),
    (64, 8, 8, 32, 257, [256, 17, 0], 16, 16, "bf16"),
    (64, 12, 3, 16, 300, [300, 299, 5], 65, 7, "bf16"),
    (32, 4, 4, 16, 100, [100, 0, 47], 8, 8, "bf16"),
    (32, 5, 1, 128, 40, [40, 3, 0], 33, 0, "bf16"),
    (256, 8, 1, 64, 400, [400, 0, 65], 20, 20, "f32"),
    (128, 4, 4, 16, 90, [90, 16, 17], 3, 40, "f32"),
    (64, 8, 8, 32, 257, [257, 0, 100], 16, 16, "f32"),
    (32, 4, 2, 64, 33, [33, 32, 1], 1, 0, "f32"),
    # many blocks of 16 rows, then enough work for those of 128: every head dim, ragged stages, a last block of few rows
    (256, 8, 1, 64, 2500, [2500, 0, 1999], 50, 50, "bf16"),
    (256, 8, 1, 16, 3001, [2977, 65, 64], 41, 0, "bf16"),
    (128, 16, 4, 128, 1100, [1100, 129, 1000], 100, 130, "bf16"),
    (64, 12, 3, 16, 900, [900, 899, 5], 100, 7, "bf16"),
    (32, 4, 4, 32, 2000, [2000, 1, 1025], 128, 8, "bf16"),
    (256, 8, 1, 64, 4100, [4100, 0, 1999], 50, 50, "bf16"),
    (256, 8, 1, 16, 5001, [4977, 65, 64], 41, 0, "bf16"),
    (64, 12, 3, 16, 1400, [1400, 1399, 5], 100, 7, "bf16"),
    (32, 4, 4, 32, 3200, [3200, 1, 1025], 128, 8, "bf16"),
    # and more keys than blocks of 32 rows would walk
    (256, 8, 1, 64, 7800, [7800, 0, 1999], 50, 50, "bf16"),
    (256, 8, 1, 16, 9201, [9177, 65, 64], 41, 0, "bf16"),
    (64, 12, 3, 16, 2601, [2601, 2599, 5], 100, 7, "bf16"),
    (32, 4, 4, 32, 6300, [6300, 1, 1025], 128, 8, "bf16"),
    # blocks of 32 rows: every head dim, an odd last block, two key ranges
    (256, 8, 1, 128, 300, [300, 0, 77], 120, 33, "bf16"),
    (128, 16, 4, 32, 333, [333, 31, 200], 60, 0, "bf16"),
    (64, 12, 3, 64, 301, [301, 299, 1], 85, 85, "bf16"),
    (32, 6, 3, 16, 129, [129, 0, 128], 130, 7, "bf16"),
    (128, 4, 4, 64, 4100, [4100, 0, 4099], 100, 1, "bf16"),
    (64, 8, 8, 16, 4097, [4097, 33, 2000], 65, 16, "bf16"),
]


@pytest.mark.parametrize("hd,nq,nkv,block,cap,lens,rows,n_self,dtype", ATTEND)
def test_attention(hd, nq, nkv, block, cap, lens, rows, n_self, dtype):
    r = np.random.default_rng(hd + cap + rows)
    c = _draw_cache(r, 5, nkv, cap, hd, block, lens + [cap, 0])
    for x in ("k", "v"):  # what lies behind a sequence's end is never read as a value
        for s in range(5):
            c[x][s, :, c["len"][s]:] = 0x7F
    g = _upload(c)
    # padded batch: an index of no sequence, a sequence twice, one of the empty ones
    want = _attend(g, c, r, dtype, nq, rows, n_self, 6, seq=[2, 0, -1, 1, 0, 4])
    assert np.all(want[2] == 0)
    _attend(g, c, r, dtype, nq, rows, n_self, 5, scale=0.05, packed=True)
    _same(g, c)


@pytest.mark.parametrize("hd,nq,nkv,block,cap,lens,rows,n_self,dtype", ATTEND[:1] + ATTEND[2:9:2] + ATTEND[9:13] + ATTEND[13:16] + ATTEND[18::2])
def test_accumulated_weights(hd, nq, nkv, block, cap, lens, rows, n_self, dtype):
    r = np.random.default_rng(hd + cap + rows + 1)
    c = _draw_cache(r, 4, nkv, cap, hd, block, lens + [cap])
    before = c["w"].astype(np.float64)
    g = _upload(c)
    seq = [3, 0, 1, 3, 2, -1]  # a sequence twice: both rows count
    _attend(g, c, r, dtype, nq, rows, n_self, 6, seq=seq, track=True)
    got = g.weight.cpu().numpy().astype(np.float64)
    added = c["w"] - before
    d = 2 * (hd + 6) * U * 64 * np.sqrt(hd) + 2.0 ** -20  # size is below 64 sqrt(hd) for these inputs (checked below)
    terms = 2 * rows * nq // nkv
    lim = (2 * d + (terms + cap + 16) * U) * added + 2 * U * c["w"] + 1e-30
    assert (np.abs(got - c["w"]) <= lim).all()
    for s in range(4):  # nothing behind a sequence's end moves
        assert np.array_equal(got[s, :, c["len"][s]:], before[s, :, c["len"][s]:])
    # twice gives twice: the order of the sums is fixed
    again = _upload({**c, "w": before})
    r2 = np.random.default_rng(9)
    _attend(again, {**co.copy(c), "w": before}, r2, dtype, nq, rows, n_self, 6, seq=seq, track=True)
    first = again.weight.clone()
    again.weight.copy_(_dev(before.astype(np.float32)))
    r2 = np.random.default_rng(9)
    _attend(again, {**co.copy(c), "w": before}, r2, dtype, nq, rows, n_self, 6, seq=seq, track=True)
    assert bool((first == again.weight).all())


def test_one_key_far_above_the_others_and_scores_that_overflow_an_exponential():
    """Scores of some thousands: the running maximum carries them; the largest key's value is the output."""
    import torch
    r = np.random.default_rng(11)
    for hd, nq, nkv, rows in ((128, 4, 2, 1), (256, 8, 1, 50), (64, 4, 4, 20)):
        c = _draw_cache(r, 1, nkv, 500, hd, 32, [500])
        k, v = _tokens(r, 1, 500, nkv, hd), _tokens(r, 1, 500, nkv, hd)
        k[0, 333] *= 64
        co.append(c, k, v, pos=[0])
        g = _upload(c)
        q = np.repeat(np.repeat(_bf16(co.values(c, 0, 0, 500)[0][333].astype(np.float32) * 4)[None, None, None], rows, 1), nq, 2)
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        g.attention(_dev(q, "bf16"), out)
        want = np.stack([co.values(c, 0, h, 500)[1][333] for h in range(nkv)])
        got = out.float().cpu().numpy()[0]
        sc = co.attention(c, q)[0][0]
        head0 = slice(0, nq // nkv)
        assert np.abs(got[:, head0] - want[0]).max() <= 2.0 ** -7 * np.abs(want[0]).max()
        assert np.abs(sc[:, head0] - want[0]).max() <= 1e-6
        assert np.isfinite(got).all()


# ---------------------------------------------------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------------------------------------------------
EVICT = [
    # hd, nkv, cap, block, lengths, keep, first
    (256, 1, 816, 64, [816, 300, 256, 257], 256, 4),
    (64, 3, 100, 16, [100, 0, 37, 99], 37, 0),
    (128, 2, 3000, 128, [3000, 2048, 1500, 1025], 1024, 1),
    (32, 2, 65, 32, [65, 64, 2, 1], 1, 1),
    (64, 1, 40, 16, [40, 39, 38, 1], 39, 5),
    (32, 1, 20000, 16, [20000, 19999, 17000, 4], 16500, 0),
    (32, 1, 40000, 32, [40000, 33000, 16385, 16384], 130, 7),
]


@pytest.mark.parametrize("hd,nkv,cap,block,lens,keep,first", EVICT)
def test_evict(hd, nkv, cap, block, lens, keep, first):
    import torch
    r = np.random.default_rng(hd + cap)
    c = co.new_cache(5, nkv, cap, hd, block, seed=cap)
    c["len"][:] = lens + [cap]
    # weights of few values: many are equal; some are NaN, infinite or of either zero
    w = r.integers(0, 30, c["w"].shape).astype(np.float32) ** 3
    for val in (np.nan, np.inf, -np.inf, -0.0, -1.5):
        w[r.random(w.shape) < 0.03] = val
    c["w"] = w
    seq = [3, 1, -1, 0, 2]
    # into another cache, its rows in another order
    d = co.new_cache(6, nkv, keep + 3, hd, block, seed=cap + 1)
    gs, gd = _upload(c), _upload(d)
    into_seq = [5, 0, 1, 3, 7]
    kept = gs.evict(keep, first=first, seq=_ints(seq), into=gd, into_seq=_ints(into_seq))
    want = co.evict(c, keep, first, seq=seq, into=d, into_seq=into_seq)
    assert np.array_equal(kept.cpu().numpy(), want)
    _same(gd, d)
    _same(gs, c)
    # in place
    kept = gs.evict(keep, first=first, seq=_ints(seq + [3]), kept=torch.empty((6, nkv, keep), dtype=torch.int32, device="cuda"))
    want = co.evict(c, keep, first, seq=seq + [3])
    assert np.array_equal(kept.cpu().numpy(), want)
    _same(gs, c)
    # again: nothing is over
    kept = gs.evict(keep, first=first, seq=_ints(seq))
    assert np.array_equal(kept.cpu().numpy(), co.evict(c, keep, first, seq=seq))
    _same(gs, c)


def test_evict_every_sequence_without_indices():
    r = np.random.default_rng(8)
    c = _draw_cache(r, 3, 2, 130, 32, 16, [130, 20, 77])
    g = _upload(c)
    kept = g.evict(50)
    assert np.array_equal(kept.cpu().numpy(), co.evict(c, 50))
    _same(g, c)


# ---------------------------------------------------------------------------------------------------------------------
# together, streams, graphs, large offsets
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("hd,nq,nkv,dtype", [(256, 8, 1, "bf16"), (64, 8, 8, "f32"), (128, 16, 4, "bf16")])
def test_a_sequences_life(hd, nq, nkv, dtype):
    """A prompt is stored, read with its weights counted, shortened; tokens are generated behind it; again."""
    r = np.random.default_rng(20)
    c = co.new_cache(4, nkv, 300, hd, 32, seed=1)
    g = _upload(c)
    seq = [2, 0]
    n = [200, 131]
    k, v = _tokens(r, 2, 200, nkv, hd, dtype=dtype), _tokens(r, 2, 200, nkv, hd, dtype=dtype)
    g.append(_dev(k, dtype), _dev(v, dtype), pos=_ints([0, 0]), count=_ints(n), seq=_ints(seq))
    co.append(c, k, v, pos=[0, 0], count=n, seq=seq)
    for turn in range(2):
        _attend(g, c, r, dtype, nq, 40, 40, 2, seq=seq, track=True)
        # the selection goes by the GPU's own sums (the oracle's, in 64 bits, may order two near ones differently)
        c["w"] = g.weight.cpu().numpy()
        kept = g.evict(100, first=2, seq=_ints(seq))
        assert np.array_equal(kept.cpu().numpy(), co.evict(c, 100, 2, seq=seq))
        for _ in range(5):
            k, v = _tokens(r, 2, 1, nkv, hd, dtype=dtype), _tokens(r, 2, 1, nkv, hd, dtype=dtype)
            g.append(_dev(k, dtype), _dev(v, dtype), seq=_ints(seq))
            co.append(c, k, v, seq=seq)
            _attend(g, c, r, dtype, nq, 1, 0, 2, seq=seq)
        _same(g, c)
        assert c["len"][[2, 0]].tolist() == [105, 105]


def test_captured_and_replayed_with_other_lengths_and_on_another_stream():
    """A decode step in a graph: positions, indices and lengths are read when it runs; eager calls live beside it."""
    import torch
    from paper_2609_34170_amd import ravel
    r = np.random.default_rng(30)
    nq, nkv, hd = 16, 4, 128
    c = _draw_cache(r, 4, nkv, 3000, hd, 64, [2900, 10, 0, 1500])
    g = _upload(c)
    seq, k = _ints([3, 0]), torch.zeros((2, 1, nkv, hd), dtype=torch.bfloat16, device="cuda")
    v, q = torch.zeros_like(k), torch.zeros((2, 1, nq, hd), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()

    def step():
        g.append(k, v, seq=seq)
        g.attention(q, out, seq=seq, track=True)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g2 = _upload(c)  # the same steps eagerly, on a stream of their own
    torch.cuda.synchronize()
    for i in range(6):
        s = [[3, 0], [1, 2], [2, 3], [0, -1], [3, 3], [1, 0]][i]
        x = [_tokens(r, *t.shape, dtype="bf16") for t in (k, v, q)]
        seq.copy_(_ints(s))
        for t, a in zip((k, v, q), x):
            t.copy_(_dev(a, "bf16"))
        graph.replay()
        co.append(c, x[0], x[1], seq=s)
        mine = torch.empty_like(q)
        kk, vv, qq, ss = _dev(x[0], "bf16"), _dev(x[1], "bf16"), _dev(x[2], "bf16"), _ints(s)
        other.wait_stream(torch.cuda.current_stream())
        g2.append(kk, vv, seq=ss, stream=other)
        g2.attention(qq, mine, seq=ss, track=True, stream=other.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out, mine)
        want, absv, size = co.attention(c, x[2], seq=s)
        lim = _bound("bf16", hd, 3000, want, absv, size)
        assert (np.abs(out.float().cpu().numpy() - want) <= lim).all()
    assert torch.equal(g.weight, g2.weight)
    c["w"] = g.weight.cpu().numpy()
    _same(g, c)
    _same(g2, c)


def test_offsets_past_32_bits():
    """A sequence of 2^24 tokens of 256 dims (4 GiB of keys), and a second one behind it: the last tokens carry the softmax."""
    import torch
    from paper_2609_34170_amd import ravel
    cap, hd, nq = 1 << 24, 256, 8
    g = ravel.Cache.empty(2, 1, cap, hd, block=128, weight=True)
    r = np.random.default_rng(40)
    k, v = _tokens(r, 2, 5, 1, hd, dtype="bf16"), _tokens(r, 2, 5, 1, hd, dtype="bf16")
    pos = _ints([cap - 5, cap - 5])
    g.append(_dev(k, "bf16"), _dev(v, "bf16"), pos=pos)
    assert g.length.tolist() == [cap, cap]
    small = co.new_cache(2, 1, 16, hd, 16, seed=0)
    co.append(small, k, v, pos=[0, 0])
    # queries along the first of the stored keys: scores of about 90 there, 0 for the 2^24 tokens of zeros
    for rows in (1, 40):
        q = np.repeat(np.repeat(k[:, :1] * np.float32(8.0), rows, 1), nq, 2)
        q = _bf16(q / np.sqrt((k[:, :1] ** 2).sum(-1, keepdims=True)) * 11)
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        g.weight.zero_()
        g.attention(_dev(q, "bf16"), out, track=True)
        want, absv, size = co.attention(small, q)
        got = out.float().cpu().numpy()
        # the zeros' share: 2^24 exp(-top) of the sum, below 1e-6 for a top score over 31
        assert (size > 31).all()
        lim = _bound("bf16", hd, 5, want, absv, size) + 1e-6 * absv + 2 * (1 << 24) * np.exp(-31.0) * absv
        assert (np.abs(got - want) <= lim).all()
        w = g.weight[:, 0, -5:].sum(-1).cpu().numpy()
        assert np.abs(w - rows * nq).max() <= 1e-4 * rows * nq
    g.weight[:, :, -5:] += 1  # (their own weights but the first's are exp(-100) and less: 0 in 32 bits)
    kept = g.evict(7, first=1)
    assert kept[1, 0].tolist() == [0, 1] + [cap - 5 + i for i in range(5)]
    at = g.k[1, 0, 2:7].float() * g.k_scale[1, 0, 0]
    assert torch.equal(at.cpu(), torch.from_numpy(co.values(small, 1, 0, 5)[0]).float())
    del g
    torch.cuda.empty_cache()


def test_the_binding_refuses_tensors_that_do_not_fit():
    import torch
    from paper_2609_34170_amd import ravel
    g = ravel.Cache.empty(2, 2, 64, 64, block=16)
    q = torch.zeros((2, 3, 4, 64), dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16, device="cuda")
    i32 = torch.zeros(2, dtype=torch.int32, device="cuda")
    for call in (lambda: g.attention(q, q.float()), lambda: g.attention(q[..., :32], q[..., :32]),
                 lambda: g.attention(q, torch.empty_like(q), kv), lambda: g.attention(q, torch.empty_like(q), kv, kv.float()),
                 lambda: g.attention(q, torch.empty_like(q), seq=i32.long()), lambda: g.attention(q, torch.empty_like(q), seq=i32[:1]),
                 lambda: g.attention(q, torch.empty_like(q).cpu()), lambda: g.attention(q.half(), torch.empty_like(q).half()),
                 lambda: g.append(kv, kv.float()), lambda: g.append(kv[:, :, :1], kv[:, :, :1]),
                 lambda: g.append(kv, kv, pos=i32.cpu()), lambda: g.append(kv.transpose(2, 3), kv.transpose(2, 3)),
                 lambda: g.evict(4, kept=torch.zeros((2, 2, 5), dtype=torch.int32, device="cuda")),
                 lambda: ravel.Cache(g.k, g.v, g.k_scale, g.v_scale[:, :, :1], g.length, 16)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ravel.RavelError, match="E_INVALID"):
        g.evict(4)  # no weights
    with pytest.raises(ravel.RavelError, match="E_INVALID"):
        g.attention(q, torch.empty_like(q), track=True)
    with pytest.raises(ravel.RavelError, match="E_SHAPE"):
        g.attention(q[:, :, :3], torch.empty_like(q[:, :, :3]))
