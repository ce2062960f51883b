"""What the cache's entry points refuse: every check answers on the host, before anything is launched."""

import ctypes
import os

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34170_amd", "libravel.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libravel.so not built")

P = 1 << 20  # an aligned address that is never read
INVALID, SHAPE = -1, -4


def _cache(**kw):
    from paper_2609_34170_amd import ravel
    d = dict(n_seq=2, n_kv_heads=2, head_dim=64, capacity=100, block=32, reserved=0, k=P, v=2 * P, k_scale=P, v_scale=P,
             len=4 * P, weight=P)
    d.update(kw)
    return ravel.RavelCache(**d)


def _lib():
    from paper_2609_34170_amd import ravel
    return ravel.load_library()


BAD_CACHES = [(dict(n_seq=0), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(head_dim=96), SHAPE), (dict(head_dim=512), SHAPE),
              (dict(capacity=0), SHAPE), (dict(capacity=(1 << 24) + 1), SHAPE), (dict(block=8), INVALID),
              (dict(block=48), INVALID), (dict(reserved=1), INVALID), (dict(k=None), INVALID), (dict(v=P + 8), INVALID),
              (dict(k_scale=None), INVALID), (dict(len=None), INVALID), (dict(v_scale=P + 2), INVALID)]


def _append(cache, batch=2, seq=None, pos=P, count=None, n=4, dtype=1, k=P, v=P, st=(512, 128, 64)):
    return _lib().ravel_cache_append(None if cache is None else ctypes.byref(cache), batch, seq, pos, count, n, dtype, k, v,
                                     *st, None)


def _query(**kw):
    from paper_2609_34170_amd import ravel
    d = dict(dtype=1, batch=2, n_q_heads=4, rows=3, n_self=3, track=0, scale=0.125, reserved=0, seq=None, q=P, self_k=P,
             self_v=P, out=P, q_stride=(1024, 256, 64), self_stride=(1024, 128, 64), out_stride=(1024, 256, 64),
             workspace=P, workspace_bytes=1 << 30)
    d.update(kw)
    return ravel.RavelCacheQuery(**d)


def _attend(cache, q):
    return _lib().ravel_cache_attention(None if cache is None else ctypes.byref(cache), None if q is None else ctypes.byref(q),
                                        None)


def _evict(cache, batch=2, seq=None, keep=10, first=0, into=None, into_seq=None, kept=P, ws=P, nbytes=1 << 30):
    return _lib().ravel_cache_evict(None if cache is None else ctypes.byref(cache), batch, seq, keep, first,
                                    None if into is None else ctypes.byref(into), into_seq, kept, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches(kw, status):
    c = _cache(**kw)
    assert _append(c) == status
    assert _lib().ravel_last_error()
    assert _attend(c, _query()) == status
    assert _evict(c) == status
    assert _evict(_cache(k=64 * P, v=65 * P), into=c) == status


def test_null_structs():
    assert _append(None) == INVALID and _attend(None, _query()) == INVALID and _evict(None) == INVALID
    assert _attend(_cache(), None) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), SHAPE), (dict(batch=32768), SHAPE), (dict(n=-1), SHAPE), (dict(n=101), SHAPE), (dict(dtype=2), INVALID),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=P + 8), INVALID), (dict(st=(512, 128, 60)), SHAPE),
    (dict(st=(-512, 128, 64)), SHAPE), (dict(dtype=0, st=(512, 126, 64)), SHAPE), (dict(seq=P + 2), INVALID),
    (dict(pos=P + 1), INVALID), (dict(count=4 * P), INVALID)])
def test_append(kw, status):
    assert _append(_cache(), **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), SHAPE), (dict(batch=40000), SHAPE), (dict(dtype=7), INVALID), (dict(n_q_heads=3), SHAPE),
    (dict(n_q_heads=0), SHAPE), (dict(rows=0), SHAPE), (dict(rows=1 << 21), SHAPE), (dict(n_self=-1), SHAPE),
    (dict(n_q_heads=1 << 14, rows=1 << 20), SHAPE), (dict(reserved=1), INVALID), (dict(q=None), INVALID),
    (dict(out=None), INVALID), (dict(self_k=None), INVALID), (dict(self_v=None), INVALID), (dict(q=P + 4), INVALID),
    (dict(out=P + 8), INVALID), (dict(self_v=P + 2), INVALID), (dict(q_stride=(1024, 255, 64)), SHAPE),
    (dict(self_stride=(1024, 128, -64)), SHAPE), (dict(out_stride=(1 << 62, 256, 64)), SHAPE), (dict(seq=P + 1), INVALID)])
def test_attention(kw, status):
    assert _attend(_cache(), _query(**kw)) == status


def test_attention_track_needs_weights_and_a_workspace():
    assert _attend(_cache(weight=None), _query(track=1)) == INVALID
    n = ctypes.c_int64(0)
    c, q = _cache(), _query(track=1, workspace_bytes=0)
    assert _lib().ravel_cache_attention_workspace(ctypes.byref(c), ctypes.byref(q), ctypes.byref(n)) == 0
    assert n.value > 0
    assert _attend(c, q) == INVALID and b"workspace of %d bytes" % n.value in _lib().ravel_last_error()
    assert _attend(c, _query(track=1, workspace_bytes=n.value - 1)) == INVALID
    assert _attend(c, _query(track=1, workspace=None, workspace_bytes=n.value)) == INVALID
    assert _attend(c, _query(track=1, workspace=P + 16, workspace_bytes=n.value)) == INVALID
    assert _lib().ravel_cache_attention_workspace(ctypes.byref(c), ctypes.byref(q), None) == INVALID


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), SHAPE), (dict(keep=0), SHAPE), (dict(keep=(1 << 24) + 1), SHAPE), (dict(first=-1), SHAPE),
    (dict(first=11), SHAPE), (dict(kept=None), INVALID), (dict(kept=P + 1), INVALID), (dict(ws=None), INVALID),
    (dict(ws=P + 16), INVALID), (dict(nbytes=0), INVALID), (dict(into_seq=P), INVALID)])
def test_evict(kw, status):
    assert _evict(_cache(), **kw) == status


def test_evict_destinations():
    far = dict(k=64 * P, v=65 * P)
    assert _evict(_cache(weight=None)) == INVALID
    for kw in (dict(head_dim=32), dict(n_kv_heads=1), dict(block=64), dict(capacity=9)):
        assert _evict(_cache(), into=_cache(**{**far, **kw})) == SHAPE, kw
    assert _evict(_cache(), into=_cache()) == INVALID  # the same memory
    assert _evict(_cache(), into=_cache(k=64 * P, v=P + 4096)) == INVALID  # part of it


def test_empty_batches_do_nothing():
    assert _append(_cache(), batch=0, k=None, v=None) == 0
    assert _attend(_cache(), _query(batch=0, q=None, out=None)) == 0
    assert _evict(_cache(), batch=0, kept=None) == 0


def test_structs_match_the_header():
    import re
    from paper_2609_34170_amd import ravel
    text = open(os.path.join(os.path.dirname(LIB), "..", "include", "ravel.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    kinds = {"int32_t": ctypes.c_int32, "float": ctypes.c_float, "int64_t": ctypes.c_int64}
    for name, st in (("ravel_cache", ravel.RavelCache), ("ravel_cache_query", ravel.RavelCacheQuery)):
        body = re.search(r"typedef struct\s*\{([^}]*)\}\s*" + name + r"\s*;", text).group(1)
        got = [(t, star, n, dim) for t, star, n, dim in re.findall(r"((?:const )?\w+)(\*?)\s+(\w+)(\[3\])?\s*;", body)]
        assert [n for _, _, n, _ in got] == [f[0] for f in st._fields_]
        for (t, star, n, dim), (_, ct) in zip(got, st._fields_):
            want = ctypes.c_void_p if star else kinds[t]
            assert ct is (want * 3 if dim else want) or (dim and ct._type_ is want and ct._length_ == 3), n


def test_indices_in_the_lengths():
    """The lengths move while rows still read their indices; only pos == len has a meaning."""
    c = _cache()
    assert _append(c, seq=4 * P) == INVALID and _append(c, seq=4 * P + 4) == INVALID
    assert _append(c, pos=4 * P + 4) == INVALID and _append(c, pos=4 * P - 4) == INVALID
    assert _append(c, count=4 * P - 4) == INVALID


def test_attention_scales_and_out():
    for scale in (-0.125, float("inf"), float("nan")):
        assert _attend(_cache(), _query(scale=scale)) == INVALID
        assert b"scale" in _lib().ravel_last_error()
    assert _attend(_cache(), _query()) == INVALID and b"out" in _lib().ravel_last_error()  # out is q


def test_evict_destinations_share_nothing():
    far = dict(k=64 * P, v=65 * P, k_scale=66 * P, v_scale=67 * P, len=68 * P, weight=69 * P)
    for kw in (dict(k_scale=P), dict(v_scale=P + 4), dict(len=4 * P + 4), dict(weight=P + 1596), dict(weight=2 * P)):
        assert _evict(_cache(), into=_cache(**{**far, **kw})) == INVALID, kw
        assert b"share memory" in _lib().ravel_last_error()


def test_the_binding_needs_a_gpu():
    import torch
    from paper_2609_34170_amd import ravel
    g = ravel.Cache.empty(2, 1, 20, 32, block=16, weight=True, device="cpu")
    x = torch.zeros((2, 1, 1, 32))
    for call in (lambda: g.append(x, x), lambda: g.attention(x, torch.empty_like(x)), lambda: g.evict(3)):
        with pytest.raises(ValueError, match="GPU"):
            call()
