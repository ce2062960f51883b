"""Cross attention with its gradients on the GPU against the 64-bit definition (tests/layer_oracle.py has the bounds)."""

import numpy as np
import pytest

from tests import layer_oracle as lo
from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


def _dev(x, dtype):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _ints(x):
    import torch
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def _near(got, want, tol, name):
    got = got.detach().float().cpu().numpy().astype(np.float64)
    bad = ~((np.abs(got - want) <= tol) | (got == want))
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


def _case(dtype, heads, B, R, K, q_len=None, k_len=None, scale=None, seed=0, spread=0.5):
    nq, nkv, hd = heads
    r = np.random.default_rng(seed + R * 31 + K + hd)
    n = lambda *s: lo.held(r.standard_normal(s) * np.exp(spread * r.standard_normal(s[-1])), dtype)  # noqa: E731
    return dict(q=n(B, R, nq, hd), k=n(B, K, nkv, hd), v=n(B, K, nkv, hd), q_len=q_len, k_len=k_len, scale=scale,
                dout=n(B, R, nq, hd), dtype=dtype)


def _run(c, poison=True, layout="plain"):
    """Through the binding; keys and rows behind the lengths hold NaN and infinities."""
    import torch
    from paper_2609_34170_amd import ravel
    x = {n: c[n].copy() for n in ("q", "k", "v", "dout")}
    if poison:
        for b in range(len(x["q"])):
            n, r = lo._len(c["k_len"], b, x["k"].shape[1]), lo._len(c["q_len"], b, x["q"].shape[1])
            x["k"][b, n:], x["v"][b, n:] = np.nan, np.inf
            x["q"][b, r:], x["dout"][b, r:] = -np.inf, np.nan
    t = {n: _dev(v, c["dtype"]) for n, v in x.items()}
    if layout == "packed":  # keys and values of one projection, sequence first
        B, K, h, d = t["k"].shape
        kv = torch.stack([t["k"], t["v"]], 2).permute(1, 0, 2, 3, 4).contiguous()  # [K, B, 2, h, d]
        t["k"], t["v"] = kv[:, :, 0].transpose(0, 1), kv[:, :, 1].transpose(0, 1)
        t["q"] = t["q"].transpose(1, 2).contiguous().transpose(1, 2)  # heads first
    ql, kl = _ints(c["q_len"]), _ints(c["k_len"])
    B, R, nq, _ = t["q"].shape
    lse = torch.full((B, nq, R), 7.0, device="cuda")
    out = ravel.cross_attention(t["q"], t["k"], t["v"], ql, kl, c["scale"], lse=lse)
    d = ravel.cross_attention_grad(t["q"], t["k"], t["v"], out, lse, t["dout"], ql, kl, c["scale"])
    torch.cuda.synchronize()
    return t, (ql, kl), {"out": out, "lse": lse, "dq": d[0], "dk": d[1], "dv": d[2]}


def _compare(c, got):
    want, tol = lo.attention(c["q"], c["k"], c["v"], c["q_len"], c["k_len"], c["scale"], c["dtype"], dout=c["dout"])
    for n in want:
        _near(got[n], want[n], tol[n], n)


TINY, SMALL, PI, LARGE, WIDE, ODD = (4, 4, 32), (8, 8, 64), (8, 1, 256), (16, 4, 128), (12, 3, 64), (10, 2, 128)


@pytest.mark.parametrize("dtype,heads,B,R,K,q_len,k_len", [
    ("bf16", TINY, 1, 1, 1, None, None),
    ("f32", TINY, 2, 3, 5, [3, 1], [0, 5]),
    ("bf16", PI, 3, 50, 16, None, None),
    ("bf16", PI, 2, 50, 33, [50, 17], [33, 1]),
    ("f32", PI, 2, 9, 40, None, [40, 17]),
    ("bf16", LARGE, 2, 100, 300, [100, 0], [299, 300]),
    ("bf16", LARGE, 1, 1, 4097, None, None),
    ("bf16", LARGE, 3, 1, 1000, None, [1000, 0, 129]),
    ("f32", LARGE, 1, 1, 700, None, None),
    ("f32", LARGE, 2, 33, 65, [33, 20], [64, 65]),
    ("bf16", WIDE, 2, 129, 257, None, [257, 128]),
    ("f32", WIDE, 1, 17, 129, None, None),
    ("bf16", ODD, 2, 27, 64, None, [63, 64]),  # rows of five heads end inside tiles
    ("bf16", ODD, 1, 300, 16, [299], None),
    ("f32", ODD, 1, 70, 31, None, None),
    ("bf16", SMALL, 2, 16, 257, None, [2, 257]),
    ("bf16", TINY, 1, 2000, 3, None, None),
    ("bf16", PI, 1, 1, 3000, None, None),
    ("bf16", PI, 1, 4, 500, None, [-3]),
    ("f32", SMALL, 1, 5, 9, [9], [100]),  # lengths beyond the tensors
    ("bf16", (2, 1, 64), 1, 700, 700, None, None),
])
def test_forward_and_gradients(dtype, heads, B, R, K, q_len, k_len):
    c = _case(dtype, heads, B, R, K, q_len, k_len)
    _, _, got = _run(c)
    _compare(c, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128, 256])
def test_heads_that_fill_the_chip(hd, dtype):
    """Blocks of the most rows and keys, in the forward and both gradients, with lengths that end inside their tiles."""
    c = _case(dtype, (8, 4, hd), 16, 201, 391, [201, 0, 130, 65, 64, 1, 33, 200] * 2, [391, 100, 0, 1, 65, 128, 129, 385] * 2)
    _, _, got = _run(c)
    _compare(c, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_tensors(dtype):
    c = _case(dtype, ODD, 2, 21, 70, [21, 8], [70, 33])
    _, _, plain = _run(c)
    _, _, got = _run(c, layout="packed")
    for n in got:
        assert (got[n] == plain[n]).all(), n
    _compare(c, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Rows whose softmax has one key, and running maxima that move far between tiles."""
    c = _case(dtype, (4, 2, 64), 1, 40, 300, scale=1.0, spread=0.0)
    c["k"] = lo.held(c["k"] * np.linspace(0.1, 5, 300)[None, :, None, None], dtype)
    _, _, got = _run(c)
    _compare(c, got)


def test_scale_zero_is_the_mean():
    c = _case("bf16", SMALL, 1, 20, 50, scale=0.0)
    _, _, got = _run(c)
    _compare(c, got)
    assert (got["dq"] == 0).all() and (got["dk"] == 0).all()


def test_no_keys_no_rows_no_batch():
    import torch
    from paper_2609_34170_amd import ravel
    z = lambda *s: torch.full(s, 3.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, k = z(2, 5, 4, 32), z(2, 0, 2, 32)
    lse = torch.empty((2, 4, 5), device="cuda")
    out = ravel.cross_attention(q, k, k, lse=lse)
    assert (out == 0).all() and (lse == -float("inf")).all()
    dq, dk, dv = ravel.cross_attention_grad(q, k, k, out, lse, q)
    assert (dq == 0).all() and dk.shape == k.shape
    q, k = z(2, 0, 4, 32), z(2, 6, 2, 32)
    lse = torch.empty((2, 4, 0), device="cuda")
    out = ravel.cross_attention(q, k, k, lse=lse)
    dq, dk, dv = ravel.cross_attention_grad(q, k, k, out, lse, q)
    assert out.shape == q.shape and (dk == 0).all() and (dv == 0).all()
    q, k = z(0, 3, 4, 32), z(0, 6, 2, 32)
    lse = torch.empty((0, 4, 3), device="cuda")
    out = ravel.cross_attention(q, k, k, lse=lse)
    assert ravel.cross_attention_grad(q, k, k, out, lse, q)[1].shape == k.shape


@pytest.mark.parametrize("heads,R,K", [(PI, 50, 16), (LARGE, 64, 400), (LARGE, 1, 900)])
def test_gradients_one_at_a_time(heads, R, K):
    import torch
    from paper_2609_34170_amd import ravel
    c = _case("bf16", heads, 2, R, K, None, [K, K // 2])
    t, (ql, kl), got = _run(c)
    args = (t["q"], t["k"], t["v"], got["out"], got["lse"], t["dout"], ql, kl)
    dq, dk, dv = ravel.cross_attention_grad(*args, need_kv=False)
    assert dk is None and dv is None and torch.equal(dq, got["dq"])
    dq, dk, dv = ravel.cross_attention_grad(*args, need_q=False)
    assert dq is None and torch.equal(dk, got["dk"]) and torch.equal(dv, got["dv"])


def test_outputs_keep_to_their_places():
    """Gradients written into one interleaved tensor leave the rest of it alone."""
    import torch
    from paper_2609_34170_amd import ravel
    c = _case("bf16", ODD, 2, 21, 70, [21, 8], [70, 33])
    t, (ql, kl), got = _run(c)
    B, K, h, d = t["k"].shape
    dkv = torch.full((B, K + 1, 3, h, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    dq = torch.full((B, 22, 10, d + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    ravel.cross_attention_grad(t["q"], t["k"], t["v"], got["out"], got["lse"], t["dout"], ql, kl, dq=dq[:, :21, :, :d],
                               dk=dkv[:, :K, 0, :, :d], dv=dkv[:, :K, 2, :, :d])
    assert torch.equal(dq[:, :21, :, :d], got["dq"]) and torch.equal(dkv[:, :K, 0, :, :d], got["dk"])
    assert torch.equal(dkv[:, :K, 2, :, :d], got["dv"])
    assert (dkv[:, :, 1] == 7).all() and (dkv[:, K] == 7).all() and (dkv[..., d:] == 7).all()
    assert (dq[:, 21] == 7).all() and (dq[..., d:] == 7).all()


def test_keys_shared_by_broadcast():
    """One context for every batch row and KV head, by strides of 0."""
    from paper_2609_34170_amd import ravel
    c = _case("bf16", SMALL, 3, 12, 40)
    c["k"][:], c["v"][:] = c["k"][:1, :, :1], c["v"][:1, :, :1]
    t, _, got = _run(c)
    k, v = (t[n][:1, :, :1].expand(t[n].shape) for n in "kv")
    assert (ravel.cross_attention(t["q"], k, v) == got["out"]).all()
    _compare(c, got)


def test_values_that_are_not_finite_reach_only_who_sees_them():
    import torch
    c = _case("bf16", SMALL, 2, 12, 40, None, [40, 20])
    _, _, plain = _run(c, poison=False)
    c["v"][0, 3, 2, 5] = np.inf
    c["q"][0, 4, 1] = np.nan
    _, _, got = _run(c, poison=False)
    out = got["out"].float()
    assert torch.isinf(out[0, :, 2, 5]).all() and torch.isnan(out[0, 4, 1]).all()
    same = torch.ones_like(out, dtype=torch.bool)
    same[0, :, 2, 5], same[0, 4, 1] = False, False
    assert (out[same] == plain["out"].float()[same]).all()
    assert (got["dq"][1] == plain["dq"][1]).all() and (got["dk"][1] == plain["dk"][1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 150])
def test_a_single_key_has_no_stride(dtype, rows):
    """The stride of a dimension with one index says nothing; values that are not finite meet no 0 that they are not given."""
    import torch
    from paper_2609_34170_amd import ravel
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    q, dout = (torch.randn(2, rows, 4, 64, device="cuda").to(t) for _ in range(2))
    k, v = (torch.randn(2, 1, 2, 64, device="cuda").to(t) for _ in range(2))
    v[1, 0, 1, 5] = float("inf")
    odd = [x.as_strided(x.shape, (128, 0, 64, 1)) for x in (k, v)]
    lse = torch.empty(2, 4, rows, device="cuda")
    out, other = ravel.cross_attention(q, k, v, lse=lse), ravel.cross_attention(q, *odd)
    assert torch.equal(out, other)
    # p = exp2(s cs - m) with m = s cs rounded, |s| < 2^7: 1 within 2^-16, divided by itself but for 3 roundings
    want = v.repeat_interleave(2, 2).expand_as(out)
    assert torch.equal(out, want) if dtype == "bf16" else torch.allclose(out, want, rtol=2.0 ** -21, atol=0)
    grads = [ravel.cross_attention_grad(q[:1], a[:1], b[:1], out[:1], lse[:1], dout[:1]) for a, b in ((k, v), odd)]
    for x, y in zip(*grads):
        assert torch.equal(x, y) and bool(torch.isfinite(x).all())


def test_offsets_beyond_32_bits():
    """Keys, values and their gradients of more than 2^31 elements; the weight lies on keys at both ends and between."""
    import torch
    from paper_2609_34170_amd import ravel
    K, hd, at = (1 << 23) + 77, 256, [3, 1 << 22, (1 << 23) - 1, (1 << 23) + 76]
    q = torch.ones(1, 1, 1, hd, device="cuda", dtype=torch.bfloat16)
    k = torch.zeros(1, K, 1, hd, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    r = torch.Generator(device="cuda").manual_seed(5)
    for i, n in enumerate(at):
        k[0, n] = 1.5 + 0.0625 * i  # scores 24 + i against 0: all weight but 2^23 e^-24 (3e-4)
        v[0, n] = torch.randn(1, hd, generator=r, device="cuda").bfloat16()
    dout = torch.randn(1, 1, 1, hd, generator=r, device="cuda").bfloat16()
    lse = torch.empty(1, 1, 1, device="cuda")
    out = ravel.cross_attention(q, k, v, lse=lse)
    dq, dk, dv = ravel.cross_attention_grad(q, k, v, out, lse, dout)
    s = torch.tensor([24.0 + i for i in range(4)], dtype=torch.float64)
    p = s.exp() / (s.exp().sum() + (K - 4))
    near, d = v[0, at, 0].double().cpu(), dout.double().cpu().view(hd)
    want = p @ near
    # probabilities and results are rounded once each (2^-8 relative)
    tol = 2.0 ** -8 * (p @ near.abs()) + 2.0 ** -8 * want.abs() + 1e-5
    assert ((out.double().cpu().view(hd) - want).abs() <= tol).all()
    assert ((dv[0, at, 0].double().cpu() - p[:, None] * d).abs() <= 2.0 ** -7 * p[:, None] * d.abs() + 1e-7).all()
    # ds = p (dout v - dout out) / 16 with out as it was rounded
    ds = p * (near @ d - out.double().cpu().view(hd) @ d) / 16
    assert ((dk[0, at, 0].double().cpu() - ds[:, None]).abs() <= 2.0 ** -6 * ds.abs()[:, None] + 1e-5).all()
    others = torch.ones(K, dtype=torch.bool, device="cuda")
    others[at] = False
    assert float(dv[0, others].abs().max()) <= 1e-9 and bool(torch.isfinite(dq).all())
