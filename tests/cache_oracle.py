"""The 8-bit key/value cache in numpy, from its definition: codes and scales exactly, attention in 64 bits.

A cache is a dict of arrays: ``k``, ``v`` uint8 codes ``[n_seq, nkv, cap, hd]``, ``ks``, ``vs`` float32
``[n_seq, nkv, ceil(cap / block)]``, ``len`` int32 ``[n_seq]``, ``w`` float32 ``[n_seq, nkv, cap]``; plus ``block``.
"""

import math

import numpy as np


def _decode_table():
    t = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        t[c] = math.nan if (c & 127) == 127 else (-x if c & 128 else x)
    return t


DECODE = _decode_table()
POSITIVE = DECODE[:127]  # ascending, 0 .. 448


def encode(x):
    """Nearest e4m3 code of float64 values, halves to the even code; infinities saturate, NaN is 0x7F (sign kept)."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.clip(np.searchsorted(POSITIVE, a), 1, 126)  # POSITIVE[hi - 1] < a <= POSITIVE[hi], or a = 0
    lo = hi - 1
    up, down = POSITIVE[hi] - a, a - POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(x), 0x7F, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_for(x):
    """The smallest power of two, 2^-100 at least, by which the largest finite magnitude of x is within 448."""
    a = np.abs(np.asarray(x, dtype=np.float64))
    a = a[np.isfinite(a)]
    top, e = (a.max() if a.size else 0.0), -100
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def new_cache(n_seq, nkv, cap, hd, block, seed=0):
    """Full of stale finite codes, scales and weights; every sequence empty."""
    r = np.random.default_rng(seed)
    nb = -(-cap // block)
    code = lambda: r.integers(0, 127, (n_seq, nkv, cap, hd), dtype=np.uint8) | (  # noqa: E731
        r.integers(0, 2, (n_seq, nkv, cap, hd), dtype=np.uint8) << 7)
    return dict(k=code(), v=code(), ks=np.exp2(r.integers(-9, -4, (n_seq, nkv, nb))).astype(np.float32),
                vs=np.exp2(r.integers(-9, -4, (n_seq, nkv, nb))).astype(np.float32), len=np.zeros(n_seq, np.int32),
                w=r.random((n_seq, nkv, cap), dtype=np.float32), block=block)


def copy(c):
    return {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in c.items()}


def _rows(c, seq, batch):
    """(row, sequence) of the rows that take part, the first of each sequence."""
    seen = set()
    for b in range(batch):
        q = b if seq is None else int(seq[b])
        if 0 <= q < len(c["len"]) and q not in seen:
            seen.add(q)
            yield b, q


def append(c, k, v, pos=None, count=None, seq=None):
    """k, v [batch, n, nkv, hd] of 32-bit (or bf16) values."""
    cap, block = c["k"].shape[2], c["block"]
    for b, q in _rows(c, seq, len(k)):
        p = int(c["len"][q].clip(0, cap)) if pos is None else int(pos[b])
        if not 0 <= p <= cap:
            continue
        m = min(k.shape[1] if count is None else min(max(int(count[b]), 0), k.shape[1]), cap - p)
        c["len"][q] = p + m
        for codes, scales, x in ((c["k"], c["ks"], k), (c["v"], c["vs"], v)):
            for h in range(x.shape[2]):
                for blk in range(p // block, -(-(p + m) // block)):
                    b0 = blk * block
                    lo, hi = max(p, b0), min(p + m, b0 + block)
                    if lo >= hi:
                        continue
                    new = x[b, lo - p:hi - p, h].astype(np.float64)
                    s = scale_for(new)
                    s0 = float(scales[q, h, blk])
                    if lo > b0:
                        if s > s0:
                            codes[q, h, b0:lo] = encode(DECODE[codes[q, h, b0:lo]] * (s0 / s))
                        s = max(s, s0)
                    codes[q, h, lo:hi] = encode(new / s)
                    scales[q, h, blk] = s
        c["w"][q, :, p:p + m] = 0


def values(c, q, h, n):
    at = np.arange(n) // c["block"]
    return tuple(DECODE[c[x][q, h, :n]] * c[x + "s"][q, h, at].astype(np.float64)[:, None] for x in ("k", "v"))


def attention(c, q, k_self=None, v_self=None, seq=None, scale=None, track=False):
    """out [batch, rows, nq, hd] in 64 bits, and per (batch, rows, nq) what a bound on rounding errors needs: sum of
    p |v| [.., hd] and the largest scale * sum |q| |k| over the keys.  ``track`` adds to c["w"], held in 64 bits then."""
    B, T, nq, hd = q.shape
    nkv = c["k"].shape[1]
    G = nq // nkv
    scale = hd ** -0.5 if scale is None else scale
    out, absv = np.zeros(q.shape), np.zeros(q.shape)
    size = np.zeros((B, T, nq))
    if track:
        c["w"] = c["w"].astype(np.float64)
    for b in range(B):
        s = b if seq is None else int(seq[b])
        if not 0 <= s < len(c["len"]):
            continue
        n = int(c["len"][s].clip(0, c["k"].shape[2]))
        for h in range(nkv):
            k, v = values(c, s, h, n)
            if k_self is not None:
                k, v = np.concatenate([k, k_self[b, :, h]]), np.concatenate([v, v_self[b, :, h]])
            if not len(k):
                continue
            rows = q[b, :, h * G:(h + 1) * G].astype(np.float64).reshape(-1, hd)
            sc = rows @ k.T * scale
            p = np.exp(sc - sc.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, :, h * G:(h + 1) * G] = (p @ v).reshape(T, G, hd)
            absv[b, :, h * G:(h + 1) * G] = (p @ np.abs(v)).reshape(T, G, hd)
            size[b, :, h * G:(h + 1) * G] = (np.abs(rows) @ np.abs(k).T * scale).max(-1).reshape(T, G)
            if track:
                c["w"][s, h, :n] += p[:, :n].sum(0)
    return out, absv, size


def evict(c, keep, first=0, seq=None, into=None, into_seq=None, batch=None):
    """Returns kept [batch, nkv, keep]; into None: in place."""
    batch = batch if batch is not None else len(c["len"] if seq is None else seq)
    nkv, block = c["k"].shape[1], c["block"]
    kept = np.full((batch, nkv, keep), -1, np.int32)
    d = c if into is None else into
    src = copy(c)
    rows = list(_rows(c, seq, batch)) if into is None else [
        (b, b if seq is None else int(seq[b])) for b, _ in _rows(into, into_seq, batch)
        if 0 <= (b if seq is None else int(seq[b])) < len(c["len"])]
    for b, q in rows:
        to = q if into is None else (b if into_seq is None else int(into_seq[b]))
        n = int(src["len"][q].clip(0, c["k"].shape[2]))
        m = min(n, keep)
        d["len"][to] = m
        for h in range(nkv):
            w = src["w"][q, h, :n].astype(np.float64)
            w = np.where(np.isnan(w), -np.inf, w)
            nan = np.isnan(src["w"][q, h, :n])
            lead = np.arange(n) < first
            order = sorted(range(n), key=lambda i: (not lead[i], bool(nan[i]) and not lead[i], 0.0 if lead[i] else -w[i], i))
            best = np.array(order[:m], dtype=np.int64)
            at = np.full(m, -1, np.int64)
            at[best[best < m]] = best[best < m]
            at[at < 0] = np.sort(best[best >= m])
            kept[b, h, :m] = at
            d["w"][to, h, :m] = src["w"][q, h][at]
            for x in ("k", "v"):
                s = src[x + "s"][q, h].astype(np.float64)[at // block]
                codes = DECODE[src[x][q, h][at]]
                for blk in range(-(-m // block)):
                    r = slice(blk * block, min(m, (blk + 1) * block))
                    top = s[r].max()
                    d[x + "s"][to, h, blk] = top
                    same = s[r] == top
                    d[x][to, h, r] = np.where(same[:, None], src[x][q, h][at[r]], encode(codes[r] * (s[r] / top)[:, None]))
    return kept
