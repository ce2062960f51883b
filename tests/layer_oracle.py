"""A layer's operators in 64 bits from their definitions: gated residual and norm, cross attention, gated MLP, with their
gradients, and for each output a bound on what the GPU's roundings can move it by.

Roundings counted: u = 2^-24 for 32-bit operations; H(t) = eps(t) / 2 for a value that is rounded to type t (bf16 2^-8,
32 bits 2^-24).  The bounds are sums of magnitudes times the number of roundings on the way; each function says which.
"""

import math

import numpy as np

U = 2.0 ** -24
H = {"bf16": 2.0 ** -8, "f32": U}


def bf16(x):
    """64- or 32-bit values rounded to bf16 (to nearest even), as float64."""
    b = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.nan, r).astype(np.float64)


def held(x, dtype):
    return bf16(x) if dtype == "bf16" else np.asarray(x, np.float32).astype(np.float64)


# ---------------------------------------------------------------------------------------------------------------------
# gated residual and norm
# ---------------------------------------------------------------------------------------------------------------------
def mod_rows(rows, mods, group):
    return (np.arange(rows) // group) % mods


def _spread(t, at, default):
    if t is None:
        return default
    return t[None] if t.ndim == 1 else t[at]


def _gather(d, at, like):
    if like.ndim == 1:
        return d.sum(0)
    out = np.zeros((like.shape[0], d.shape[1]))
    np.add.at(out, at, d)
    return out


def residual(x, f=None, post=None, alpha=None, gate=None, group=1, eps=1e-6):
    """t and the magnitude that its roundings go by."""
    if f is None:
        return x, np.zeros_like(x)
    mods = gate.shape[0] if gate is not None and gate.ndim == 2 else 1
    F = f if post is None else f / np.sqrt((f * f).mean(-1, keepdims=True) + eps) * (1 + post)
    add = F * (1.0 if alpha is None else float(alpha)) * _spread(gate, mod_rows(len(x), mods, group), 1.0)
    return x + add, np.abs(x) + np.abs(add)


def norm(t, scale=None, shift=None, group=1, eps=1e-6):
    n = t / np.sqrt((t * t).mean(-1, keepdims=True) + eps)
    y = n * (1 + _spread(scale, mod_rows(len(t), 1 if scale is None or scale.ndim == 1 else len(scale), group), 0.0))
    b = _spread(shift, mod_rows(len(t), 1 if shift is None or shift.ndim == 1 else len(shift), group), 0.0)
    return y + b, np.abs(y) + np.abs(b)


def norm_grad(t, dy, d_out, f=None, post=None, alpha=None, gate=None, scale=None, shift=None, group=1, eps=1e-6):
    """Gradients by input, and each one's magnitude: every product and sum with absolute values in place of the terms.

    A row's sums (at most 16 elements a thread in order, then a tree) round at most 32 times, r and rf half of that and
    twice more; with the few products around them every value of a row is within 96 u of its magnitude, a sum over rows
    within 96 + rows."""
    rows = len(t)

    def rule(m):
        return mod_rows(rows, 1 if m is None or m.ndim == 1 else len(m), group)

    r = 1 / np.sqrt((t * t).mean(-1, keepdims=True) + eps)
    n = t * r
    s1 = 1 + _spread(scale, rule(scale), np.zeros((1, t.shape[1])))
    dn = dy * s1
    dt = d_out + r * (dn - n * (dn * n).mean(-1, keepdims=True))
    adt = np.abs(d_out) + r * (np.abs(dn) + np.abs(n) * np.abs(dn * n).mean(-1, keepdims=True))
    g, m = {"x": dt}, {"x": adt}
    if scale is not None:
        g["scale"], m["scale"] = _gather(dy * n, rule(scale), scale), _gather(np.abs(dy * n), rule(scale), scale)
    if shift is not None:
        g["shift"], m["shift"] = _gather(dy, rule(shift), shift), _gather(np.abs(dy), rule(shift), shift)
    if f is None:
        return g, m
    rf = 1 / np.sqrt((f * f).mean(-1, keepdims=True) + eps) if post is not None else 1.0
    mm = f * rf
    F = mm * (1 + post) if post is not None else mm
    a = 1.0 if alpha is None else float(alpha)
    ga = _spread(gate, rule(gate), np.ones((1, t.shape[1])))
    if gate is not None:
        g["gate"], m["gate"] = _gather(a * dt * F, rule(gate), gate), _gather(np.abs(a * F) * adt, rule(gate), gate)
    if alpha is not None:
        g["alpha"], m["alpha"] = (dt * ga * F).sum().reshape(1), (adt * np.abs(ga * F)).sum().reshape(1)
    dF, adF = a * ga * dt, np.abs(a * ga) * adt
    if post is not None:
        g["post"], m["post"] = (dF * mm).sum(0), (adF * np.abs(mm)).sum(0)
        dm, adm = dF * (1 + post), adF * np.abs(1 + post)
        dF = rf * (dm - mm * (dm * mm).mean(-1, keepdims=True))
        adF = rf * (adm + np.abs(mm) * (adm * np.abs(mm)).mean(-1, keepdims=True))
    g["f"], m["f"] = dF, adF
    return g, m


# ---------------------------------------------------------------------------------------------------------------------
# cross attention: q [B, R, nq, hd], k and v [B, K, nkv, hd]
# ---------------------------------------------------------------------------------------------------------------------
def _len(x, b, most):
    return most if x is None else min(max(int(x[b]), 0), most)


def attention(q, k, v, q_len=None, k_len=None, scale=None, dtype="bf16", dout=None, out_in=None):
    """dict of out, lse (and dq, dk, dv with dout), and the dict of bounds.

    A score is off by at most (hd + 6) u size, size = scale sum |q| |k| (its sum, its scaling and exponent), and so is the
    row's lse; the exponential by 2^-22: a probability by the factor d = 2 (hd + 6) u size + 2^-22.  In bf16 probabilities
    are rounded for the second product, and the scores' gradients for theirs: h = 2^-8 each.  Sums over n terms add (n +
    16) u.  D = sum dout out takes out as the call holds it (out_in), off by that output's bound e_out; dout v by (hd + 4) u
    of its magnitude.
    """
    B, R, nq, hd = q.shape
    K, nkv = k.shape[1:3]
    G, scale = nq // nkv, hd ** -0.5 if scale is None else scale
    h = H["bf16"] if dtype == "bf16" else 0.0
    hh = H[dtype]
    z = lambda *s: np.zeros(s)  # noqa: E731
    res = {"out": z(B, R, nq, hd), "lse": np.full((B, nq, R), -np.inf), "dq": z(B, R, nq, hd), "dk": z(B, K, nkv, hd),
           "dv": z(B, K, nkv, hd)}
    tol = {n: np.zeros(x.shape) for n, x in res.items()}
    for b in range(B):
        r, n = _len(q_len, b, R), _len(k_len, b, K)
        if r == 0 or n == 0:
            continue
        for j in range(nq):
            c = j // G
            qq, kk, vv = q[b, :r, j], k[b, :n, c], v[b, :n, c]
            s = scale * qq @ kk.T
            size = scale * np.abs(qq) @ np.abs(kk).T
            top = s.max(-1, keepdims=True)
            e = np.exp(s - top)
            p = e / e.sum(-1, keepdims=True)
            res["out"][b, :r, j] = p @ vv
            res["lse"][b, j, :r] = (top + np.log(e.sum(-1, keepdims=True)))[:, 0]
            big = size.max(-1, keepdims=True)  # the row's maximum is off by as much
            d = 2 * (hd + 6) * U * np.maximum(size, big) + 2.0 ** -22
            e_out = (p * (d + d.max(-1, keepdims=True) + h + (n + 16) * U)) @ np.abs(vv) + hh * np.abs(p @ vv)
            tol["out"][b, :r, j] = e_out
            tol["lse"][b, j, :r] = (d.max(-1) + (n + 16) * U + 4 * U * np.abs(res["lse"][b, j, :r]))
            if dout is None:
                continue
            do = dout[b, :r, j]
            o = p @ vv
            dp, adp = do @ vv.T, np.abs(do) @ np.abs(vv).T
            D = (do * o).sum(-1, keepdims=True)
            e_D = (np.abs(do) * e_out).sum(-1, keepdims=True) + (hd + 4) * U * np.abs(do * o).sum(-1, keepdims=True)
            d2 = d + d.max(-1, keepdims=True) + (n + 20) * U + 4 * U * np.abs(res["lse"][b, j, :r, None])
            ds = p * (dp - D)
            e_ds = p * (d2 * (np.abs(dp) + np.abs(D)) + (hd + 6) * U * adp + e_D) + h * np.abs(ds)
            res["dv"][b, :n, c] += p.T @ do
            tol["dv"][b, :n, c] += (p * (d2 + h + (G * R + 16) * U)).T @ np.abs(do)
            res["dq"][b, :r, j] = scale * ds @ kk
            tol["dq"][b, :r, j] = scale * (e_ds * (1 + h) + (n + 20) * U * np.abs(ds)) @ np.abs(kk) + hh * np.abs(res["dq"][b, :r, j])
            res["dk"][b, :n, c] += scale * ds.T @ qq
            tol["dk"][b, :n, c] += scale * (e_ds * (1 + h) + (G * R + 20) * U * np.abs(ds)).T @ np.abs(qq)
    tol["dk"] += hh * np.abs(res["dk"])
    tol["dv"] += hh * np.abs(res["dv"])
    return res, tol


# ---------------------------------------------------------------------------------------------------------------------
# gated MLP
# ---------------------------------------------------------------------------------------------------------------------
def act(x, kind):
    """Activation and slope."""
    if kind == "silu":
        s = 1 / (1 + np.exp(-x))
        return x * s, s * (1 + x * (1 - s))
    c = math.sqrt(2 / math.pi)
    # (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), which does not cancel where tanh goes to -1
    s = 1 / (1 + np.exp(np.minimum(-2 * c * (x + 0.044715 * x ** 3), 700)))
    return x * s, s + 2 * x * s * (1 - s) * c * (1 + 3 * 0.044715 * x * x)


# The activation's exponential takes an argument t that is rounded a few times (6 u |t| of its result; |t| < 90, beyond
# which the result is x or less than 2^-100 of it) and with reciprocal and products adds 10 u: 2^-15 covers 550 u.  The
# slopes' terms cancel at most against 1.13 times themselves.
ACT = 2.0 ** -15


def mlp(x, wg, wu, kind, dtype):
    """h, gate and up values, and their bounds: products of (K + 5) roundings, slope at most 1.13, one rounding at the end."""
    K = x.shape[1]
    g, u = x @ wg.T, x @ wu.T
    eg, eu = ((K + 5) * U * np.abs(x) @ np.abs(w).T for w in (wg, wu))
    a, _ = act(g, kind)
    ea = 1.13 * eg + ACT * np.abs(a)
    h = a * u
    eh = ea * np.abs(u) + (np.abs(a) + ea) * eu + 2 * U * np.abs(h)
    return {"h": h, "gate": g, "up": u}, {"h": eh + H[dtype] * (np.abs(h) + eh), "gate": eg + H[dtype] * (np.abs(g) + eg),
                                          "up": eu + H[dtype] * (np.abs(u) + eu)}


def mlp_grad(x, wg, wu, gate, up, dh, kind, dtype, weight_dtype=None):
    """dx, dwg, dwu from gate and up as they are held: the hidden gradients are rounded to dtype, sums of n terms add (n +
    16) u, one rounding at the end."""
    a, slope = act(gate, kind)
    dg, du = dh * up * slope, dh * a
    eg = 2 * ACT * np.abs(dh * up) * (1 + np.abs(gate)) + H[dtype] * np.abs(dg)
    eu = ACT * np.abs(du) + 2 * U * np.abs(du) + H[dtype] * np.abs(du)
    F, M = gate.shape[1], len(x)
    res = {"dx": dg @ wg + du @ wu, "dwg": dg.T @ x, "dwu": du.T @ x}
    n, m = (2 * F + 16) * U, (M + 16) * U
    tol = {"dx": (eg + n * np.abs(dg)) @ np.abs(wg) + (eu + n * np.abs(du)) @ np.abs(wu),
           "dwg": (eg + m * np.abs(dg)).T @ np.abs(x), "dwu": (eu + m * np.abs(du)).T @ np.abs(x)}
    for k in tol:
        t = dtype if k == "dx" else weight_dtype or dtype
        tol[k] = tol[k] + H[t] * (np.abs(res[k]) + tol[k])
    return res, tol
