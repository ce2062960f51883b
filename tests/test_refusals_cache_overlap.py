"""Calls whose arguments share memory that the call moves are refused on the host, before anything is launched."""

import ctypes

import pytest

from tests.test_refusals_cache import INVALID, LIB, P, _cache, _evict, _lib  # noqa: F401
from tests.test_refusals_cache import pytestmark  # noqa: F401

FAR = dict(k=64 * P, v=65 * P, k_scale=66 * P, v_scale=67 * P, len=68 * P, weight=69 * P)
OWN = dict(k=32 * P, v=33 * P, k_scale=34 * P, v_scale=35 * P, len=36 * P, weight=37 * P)
KEPT, WS, IDX, IDX2 = 40 * P, 48 * P, 56 * P, 57 * P


def _workspace(c, batch=2, keep=10):
    n = ctypes.c_int64(0)
    assert _lib().ravel_cache_evict_workspace(ctypes.byref(c), batch, keep, ctypes.byref(n)) == 0
    return n.value


def _refused(word, **kw):
    c = _cache(**OWN)
    args = dict(kept=KEPT, ws=WS, nbytes=_workspace(c), seq=IDX)
    args.update(kw)
    assert _evict(c, **args) == INVALID, kw
    assert word in _lib().ravel_last_error(), (kw, _lib().ravel_last_error())


def test_evict_indices_in_memory_that_the_call_moves():
    """Lengths move while rows still read their indices: in place the cache's own, otherwise the destination's."""
    into = _cache(**FAR)
    for at in (36 * P, 36 * P + 4, 36 * P - 4):
        _refused(b"seq", seq=at)
    for at in (68 * P, 68 * P + 4, 68 * P - 4):
        _refused(b"seq", into=into, seq=at, into_seq=IDX2)
        _refused(b"seq", into=into, seq=None, into_seq=at)
    for at in (KEPT, KEPT + 2 * 2 * 10 * 4 - 4, WS):
        _refused(b"seq", seq=at)
        _refused(b"seq", into=into, into_seq=at)
    for x in (37 * P, 34 * P):  # weights, scales
        _refused(b"seq", seq=x)


def test_evict_results_in_memory_that_the_call_reads():
    """The moves read the kept indices back and the workspace's notes: neither lies in a cache or in the other."""
    into = _cache(**FAR)
    for x in ("k", "v", "k_scale", "v_scale", "len", "weight"):
        _refused(b"kept", kept=OWN[x])
        _refused(b"workspace", ws=OWN[x])
        _refused(b"kept", into=into, kept=FAR[x])
        _refused(b"workspace", into=into, ws=FAR[x])
    _refused(b"kept", kept=WS)
    _refused(b"kept", kept=WS + _workspace(_cache(**OWN)) - 4)
