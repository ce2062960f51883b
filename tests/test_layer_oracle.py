"""The 64-bit definitions of a layer's operators: their gradients against central differences, and closed forms."""

import numpy as np
import pytest

from tests import layer_oracle as lo


def _difference(f, x, d, step=1e-5):
    """d/ds of f(x + s d) at 0, by differences that are exact to third order."""
    g = lambda s: f(x + s * d)  # noqa: E731
    return (8 * (g(step) - g(-step)) - (g(2 * step) - g(-2 * step))) / (12 * step)


def _check(loss, inputs, grads):
    r = np.random.default_rng(5)
    for name, x in inputs.items():
        d = r.standard_normal(x.shape)
        want = _difference(lambda y: loss({**inputs, name: y}), x, d)
        got = float((grads[name] * d).sum())
        assert abs(got - want) <= 1e-7 * (abs(want) + 1), name


@pytest.mark.parametrize("post,alpha,gate,mods,group,static", [
    (False, False, True, 6, 1, False), (True, True, True, 3, 2, False), (True, True, False, 1, 1, True), (False, True, True, 4, 1, True),
    (False, False, False, 2, 1, False)])
def test_norm_gradients(post, alpha, gate, mods, group, static):
    r = np.random.default_rng(1)
    rows, w = 6, 8
    x = dict(x=r.standard_normal((rows, w)), f=r.standard_normal((rows, w)))
    if post:
        x["post"] = 0.3 * r.standard_normal(w)
    if alpha:
        x["alpha"] = r.standard_normal(1)
    if gate:
        x["gate"] = r.standard_normal((mods, w))
    for n in ("scale", "shift"):
        x[n] = 0.3 * r.standard_normal(w if static else (mods, w))
    dy, do = r.standard_normal((rows, w)), r.standard_normal((rows, w))

    def parts(i):
        a = {n: i[n] for n in ("f", "post", "gate") if n in i}
        t, _ = lo.residual(i["x"], alpha=i["alpha"][0] if alpha else None, group=group, **a)
        return t, lo.norm(t, i["scale"], i["shift"], group)[0]

    t, _ = parts(x)
    g, _ = lo.norm_grad(t, dy, do, group=group, **{**{n: v for n, v in x.items() if n != "x"},
                                                   **({"alpha": x["alpha"][0]} if alpha else {})})
    _check(lambda i: float((parts(i)[1] * dy + parts(i)[0] * do).sum()), x, g)


@pytest.mark.parametrize("nq,nkv,q_len,k_len", [(2, 2, None, None), (4, 2, [3, 0], [5, 2]), (3, 1, None, [0, 4])])
def test_attention_gradients(nq, nkv, q_len, k_len):
    r = np.random.default_rng(2)
    x = dict(q=r.standard_normal((2, 3, nq, 4)), k=r.standard_normal((2, 5, nkv, 4)), v=r.standard_normal((2, 5, nkv, 4)))
    do = r.standard_normal((2, 3, nq, 4))
    g, _ = lo.attention(**x, q_len=q_len, k_len=k_len, dout=do)
    _check(lambda i: float((lo.attention(**i, q_len=q_len, k_len=k_len)[0]["out"] * do).sum()), x,
           {n: g["d" + n] for n in x})


def test_attention_closed_forms():
    q, k, v = np.ones((1, 2, 1, 4)), np.ones((1, 3, 1, 4)), np.arange(12.0).reshape(1, 3, 1, 4)
    out, _ = lo.attention(q, k, v)  # equal keys: the mean of the values; lse = score + log 3
    assert np.allclose(out["out"], v.mean(1, keepdims=True))
    assert np.allclose(out["lse"], 2 + np.log(3))
    out, _ = lo.attention(q, k, v, k_len=[1])
    assert np.allclose(out["out"], v[:, :1])


@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_mlp_gradients(kind):
    r = np.random.default_rng(3)
    x = dict(x=r.standard_normal((3, 4)), wg=r.standard_normal((5, 4)), wu=r.standard_normal((5, 4)))
    dh = r.standard_normal((3, 5))
    f, _ = lo.mlp(**x, kind=kind, dtype="f32")
    g, _ = lo.mlp_grad(x["x"], x["wg"], x["wu"], f["gate"], f["up"], dh, kind, "f32")
    _check(lambda i: float((lo.mlp(**i, kind=kind, dtype="f32")[0]["h"] * dh).sum()), x, {n: g["d" + n] for n in x})


def test_bf16_rounding():
    assert lo.bf16(np.array([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1.0, 0.0])).tolist() == [1.0, 1 + 2.0 ** -6, -1.0, 0.0]
