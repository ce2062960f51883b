"""Gated residual and norm with its gradients on the GPU against the 64-bit definition (tests/layer_oracle.py has the
bounds)."""

import numpy as np
import pytest

from tests import layer_oracle as lo
from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]
U = lo.U


def _dev(x, dtype="f32", pad=0):
    """On the GPU; ``pad`` columns of NaN behind every row (a strided view)."""
    import torch
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(T)
    if not pad:
        return t
    big = torch.full((t.shape[0] + 1, t.shape[1] + pad), float("nan"), dtype=T, device="cuda")
    big[:-1, :t.shape[1]] = t
    return big[:-1, :t.shape[1]]


def _out(rows, width, dtype, pad):
    import torch
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    return torch.full((rows + 1, width + pad), 7.0, dtype=T, device="cuda")[:-1, :width]


def _surroundings(t):
    """What lies behind the rows of an _out, and the row behind the last."""
    base, (r, w) = t._base, t.shape
    return base[-1, :], base[:, w:]


def _near(got, want, tol, name):
    got = got.detach().float().cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], np.broadcast_to(tol, want.shape)[bad][:4])


CASES = [
    # rows, width, stream, dtype, mods, group, what is there, pad
    (1, 8, "f32", "f32", 1, 1, "f gate scale shift", 0),
    (50, 1024, "f32", "bf16", 50, 1, "f gate scale shift", 0),
    (3, 24, "bf16", "bf16", 3, 1, "f gate scale shift post alpha", 8),
    (130, 1000, "f32", "bf16", 13, 10, "f gate scale", 8),
    (77, 256, "f32", "f32", 7, 1, "f gate scale shift alpha", 4),
    (700, 520, "f32", "bf16", 1, 1, "f post alpha scale", 16),
    (700, 128, "bf16", "bf16", 5, 3, "f post gate scale shift", 0),
    (64, 2048, "f32", "bf16", 64, 1, "f gate scale shift", 0),
    (33, 2056, "f32", "f32", 4, 9, "f gate scale shift post", 0),
    (20, 4096, "bf16", "bf16", 20, 1, "scale shift", 0),
    (21, 4104, "f32", "bf16", 2, 4, "f gate scale", 0),
    (9, 8192, "f32", "bf16", 3, 2, "f gate scale shift post alpha", 0),
    (40, 64, "f32", "bf16", 100, 1, "f gate scale shift", 0),  # modulation rows that no row uses
    (5, 136, "f32", "bf16", 2, 1000000000, "f gate scale shift", 0),  # a group longer than the rows
    (300, 72, "f32", "bf16", 1, 1, "f", 0),
    (2100, 16, "f32", "f32", 2, 1, "f gate scale shift alpha post", 0),
]


def _inputs(case, seed=0):
    rows, w, S, T, mods, group, what, pad = case
    r = np.random.default_rng(rows * 7 + w + seed)
    what = what.split()
    n = lambda *s: r.standard_normal(s)  # noqa: E731
    x = {"x": lo.held(2 * n(rows, w), S)}
    if "f" in what:
        x["f"] = lo.held(n(rows, w) * np.exp(n(rows, 1)), T)
    if "post" in what:
        x["post"] = lo.held(0.3 * n(w), "f32")
    if "alpha" in what:
        x["alpha"] = lo.held(n(1), "f32")
    for m in ("gate", "scale", "shift"):
        if m in what:
            x[m] = lo.held(0.5 * n(*((w,) if mods == 1 else (mods, w))), "f32")
    return x, lo.held(n(rows, w), T), lo.held(n(rows, w), S)


def _upload(x, case):
    import torch
    S, T, pad = case[2], case[3], case[7]
    t = {n: _dev(v, {"x": S, "f": T}.get(n, "f32"), pad if n in "xf" else 0) for n, v in x.items()}
    if "scale" in x and x["scale"].ndim == 2:  # chunks of a conditioning layer's rows
        mods, w = x["scale"].shape
        rows = torch.full((mods, 3 * w), float("nan"), device="cuda")
        for i, m in enumerate(("gate", "scale", "shift")):
            if m in t:
                rows[:, i * w:(i + 1) * w] = t[m]
                t[m] = rows[:, i * w:(i + 1) * w]
    return t


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}x{c[1]}-{c[2]}-{c[3]}-{c[4]}of{c[5]}-{c[6].replace(' ', '_')}")
def test_forward_and_gradients(case):
    import torch
    from paper_2609_34170_amd import ravel
    rows, w, S, T, mods, group, _, pad = case
    x, dy, do = _inputs(case)
    t = _upload(x, case)
    mod = {n: t.get(n) for n in ("f", "post", "alpha", "gate", "scale")}
    y = _out(rows, w, T, pad)
    x_out = _out(rows, w, S, pad) if "f" in x else None
    got_y, got_x = ravel.norm_residual(t["x"], **mod, shift=t.get("shift"), group=group, y=y, x_out=x_out)
    assert got_y is y and got_x is (x_out if "f" in x else t["x"])
    torch.cuda.synchronize()
    ins = {n: x[n] for n in ("f", "post", "gate") if n in x}
    if "alpha" in x:
        ins["alpha"] = x["alpha"][0]
    want, mag = lo.residual(x["x"], group=group, **ins)
    if "f" in x:  # F has 17 roundings of its row's sum and a few products
        _near(x_out, want, 24 * U * mag + lo.H[S] * (np.abs(want) + 24 * U * mag), "x_out")
    held = got_x.double().cpu().numpy()  # y is the norm of what x_out holds
    want_y, mag_y = lo.norm(held, x.get("scale"), x.get("shift"), group)
    _near(y, want_y, 24 * U * mag_y + lo.H[T] * (np.abs(want_y) + 24 * U * mag_y), "y")
    for o in (y, x_out):
        if o is not None:
            assert all((s == 7).all() for s in _surroundings(o))

    d = {"x": _out(rows, w, S, pad)}
    if "f" in x:
        d["f"] = _out(rows, w, T, pad)
    for n in ("post", "alpha", "gate", "scale", "shift"):
        if n in x:
            d[n] = torch.full(x[n].shape, 7.0, device="cuda")
    for again in range(2):  # the same bits every time
        g = ravel.norm_residual_grad(got_x, _dev(dy, T), _dev(do, S), **mod, group=group, grads=d)
        if again:
            assert all(torch.equal(g[n], first[n]) for n in g)
        first = {n: v.clone() for n, v in g.items()}
    want, mag = lo.norm_grad(held, dy, do, group=group, **ins, scale=x.get("scale"), shift=x.get("shift"))
    assert set(g) == set(want)
    for n in want:
        k = 96 + (0 if n in "xf" else rows + 16)
        half = lo.H[{"x": S, "f": T}.get(n, "f32")]
        _near(g[n], want[n], k * U * mag[n] + half * (np.abs(want[n]) + k * U * mag[n]), "d" + n)
    for n in ("x", "f"):
        if n in d:
            assert all((s == 7).all() for s in _surroundings(d[n]))


def test_parts_and_defaults():
    """Missing gradients count as zero, outputs that are not wanted are not needed, outputs may take their inputs' place."""
    import torch
    from paper_2609_34170_amd import ravel
    case = (37, 264, "f32", "bf16", 37, 1, "f gate scale shift alpha post", 0)
    x, dy, do = _inputs(case)
    t = _upload(x, case)
    mod = {n: t[n] for n in ("f", "post", "alpha", "gate", "scale")}
    y, x_out = ravel.norm_residual(t["x"], **mod, shift=t["shift"])
    place = t["x"].clone()
    y2, same = ravel.norm_residual(place, **mod, shift=t["shift"], x_out=place)
    assert same is place and torch.equal(place, x_out) and torch.equal(y, y2)
    full = ravel.norm_residual_grad(x_out, _dev(dy, "bf16"), _dev(do), **mod, shift=t["shift"])
    assert set(full) == {"x", "f", "post", "alpha", "gate", "scale", "shift"}
    assert full["f"].dtype is torch.bfloat16 and full["gate"].shape == t["gate"].shape
    d = _dev(do)
    part = ravel.norm_residual_grad(x_out, _dev(dy, "bf16"), d, **mod, grads={"x": d, "post": None})
    assert part["x"] is d and torch.equal(d, full["x"]) and torch.equal(part["post"], full["post"])
    for dyy, doo in ((None, do), (dy, None)):
        g = ravel.norm_residual_grad(x_out, None if dyy is None else _dev(dyy, "bf16"), None if doo is None else _dev(doo), **mod)
        z = ravel.norm_residual_grad(x_out, _dev(np.zeros_like(dy) if dyy is None else dyy, "bf16"),
                                     _dev(np.zeros_like(do) if doo is None else doo), **mod)
        assert all(torch.equal(g[n], z[n]) for n in z)


def test_no_rows():
    import torch
    from paper_2609_34170_amd import ravel
    x, f = torch.empty((0, 64), device="cuda"), torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    scale, gate = torch.randn(64, device="cuda"), torch.randn((3, 64), device="cuda")
    y, x_out = ravel.norm_residual(x, f, gate=gate, scale=scale)  # (the addresses of empty tensors are 0)
    assert y.shape == (0, 64) and x_out.shape == (0, 64)
    g = ravel.norm_residual_grad(x, f, None, f, gate=gate, scale=scale, grads={"gate": None, "scale": None})
    assert (g["gate"] == 0).all() and (g["scale"] == 0).all()


def test_values_that_are_not_finite_stay_in_their_row():
    import torch
    from paper_2609_34170_amd import ravel
    x, f = torch.randn((6, 128), device="cuda"), torch.randn((6, 128), device="cuda").bfloat16()
    scale = torch.randn(128, device="cuda")
    y0, t0 = ravel.norm_residual(x, f, scale=scale)
    x[2, 5], f[4, 7] = float("nan"), float("inf")
    y, t = ravel.norm_residual(x, f, scale=scale)
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], y0[keep]) and torch.equal(t[keep], t0[keep])
    assert torch.isnan(y[2].float()).all() and torch.isnan(y[4].float()).any()
