"""A layer's operators as they are used: the adapter and MLP halves of an expert layer with the linear layers between them,
forward and backward; captured into graphs; on other streams."""

import numpy as np
import pytest

from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]

B, H, F, W, NQ, NKV, HD, MLP = 3, 10, 5, 64, 4, 2, 32, 136  # samples, rows of each, pathway tokens, width, heads, hidden


def _parameters(seed=0):
    r = np.random.default_rng(seed)
    n = lambda s, *shape: (s * r.standard_normal(shape)).astype(np.float32)  # noqa: E731
    return dict(x=n(1, B * H, W), z=n(1, B * F, W), gamma=n(0.2, W), wq=n(W ** -0.5, NQ * HD, W), wk=n(W ** -0.5, NKV * HD, W),
                wv=n(W ** -0.5, NKV * HD, W), wo=n(W ** -0.5, W, NQ * HD), alpha=n(1, 1), mod=n(0.3, B * H, 3 * W),
                wg=n(W ** -0.5, MLP, W), wu=n(W ** -0.5, MLP, W), wd=n(MLP ** -0.5, W, MLP), gamma2=n(0.2, W)), n(1, B * H, W), n(1, B * H, W)


def _layer(p, d_y, d_x, dtype, stream=None):
    """Outputs and the gradients of sum(y d_y + x3 d_x) by the operators; every parameter is a GPU tensor."""
    from paper_2609_34170_amd import ravel
    import torch
    T = dtype
    z, lin = p["z"].to(T), {k: p[k].to(T) for k in ("wq", "wk", "wv", "wo", "wg", "wu", "wd")}
    scale, shift, gate = p["mod"][:, :W], p["mod"][:, W:2 * W], p["mod"][:, 2 * W:]
    y1, x = ravel.norm_residual(p["x"], scale=p["gamma"], y=torch.empty(p["x"].shape, dtype=T, device="cuda"))
    q = (y1 @ lin["wq"].t()).view(B, H, NQ, HD)
    k, v = ((z @ lin[n].t()).view(B, F, NKV, HD) for n in ("wk", "wv"))
    lse = torch.empty((B, NQ, H), device="cuda")
    o = ravel.cross_attention(q, k, v, lse=lse)
    f1 = o.view(B * H, -1) @ lin["wo"].t()
    y2, x2 = ravel.norm_residual(x, f1, alpha=p["alpha"], scale=scale, shift=shift)
    g, u = (torch.empty((B * H, MLP), dtype=T, device="cuda") for _ in range(2))
    h = ravel.gated_mlp(y2, lin["wg"], lin["wu"], gate=g, up=u)
    f2 = h @ lin["wd"].t()
    y3, x3 = ravel.norm_residual(x2, f2, gate=gate, scale=p["gamma2"])

    d = {}
    dmod = torch.empty((B * H, 3 * W), device="cuda")
    e = ravel.norm_residual_grad(x3, d_y.to(T), d_x, f2, gate=gate, scale=p["gamma2"],
                                 grads={"x": None, "f": None, "gate": dmod[:, 2 * W:], "scale": None})
    d["gamma2"], dx2, df2 = e["scale"], e["x"], e["f"]
    d["wd"] = df2.t() @ h
    dy2, d["wg"], d["wu"] = ravel.gated_mlp_grad(y2, lin["wg"], lin["wu"], g, u, df2 @ lin["wd"], weight_dtype=torch.float32)
    e = ravel.norm_residual_grad(x2, dy2, dx2, f1, alpha=p["alpha"], scale=scale, shift=shift,
                                 grads={"x": None, "f": None, "alpha": None, "scale": dmod[:, :W], "shift": dmod[:, W:2 * W]})
    d["alpha"], dx1, df1 = e["alpha"], e["x"], e["f"]
    d["wo"] = df1.t() @ o.view(B * H, -1)
    dq, dk, dv = ravel.cross_attention_grad(q, k, v, o, lse, (df1 @ lin["wo"]).view(o.shape))
    dq, dk, dv = (t.reshape(t.shape[0] * t.shape[1], -1) for t in (dq, dk, dv))
    d["wq"], d["wk"], d["wv"] = dq.t() @ y1, dk.t() @ z, dv.t() @ z
    d["z"] = dk @ lin["wk"] + dv @ lin["wv"]
    e = ravel.norm_residual_grad(x, dq @ lin["wq"], dx1, scale=p["gamma"])
    d["x"], d["gamma"], d["mod"] = e["x"], e["scale"], dmod
    return {"y": y3, "x3": x3}, d


def _reference(p, d_y, d_x):
    """The same in 64 bits from the definitions, by automatic differentiation."""
    import torch
    p = {n: torch.from_numpy(t).double().requires_grad_() for n, t in p.items()}
    unit = lambda t: t / torch.sqrt(t.pow(2).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    y1 = unit(p["x"]) * (1 + p["gamma"])
    heads = lambda t, r, n: t.view(B, r, n, HD).transpose(1, 2)  # noqa: E731
    q, k, v = heads(y1 @ p["wq"].t(), H, NQ), heads(p["z"] @ p["wk"].t(), F, NKV), heads(p["z"] @ p["wv"].t(), F, NKV)
    k, v = (t.repeat_interleave(NQ // NKV, 1) for t in (k, v))
    o = (torch.softmax(q @ k.transpose(2, 3) / HD ** 0.5, -1) @ v).transpose(1, 2).reshape(B * H, -1)
    x2 = p["x"] + p["alpha"] * (o @ p["wo"].t())
    y2 = unit(x2) * (1 + p["mod"][:, :W]) + p["mod"][:, W:2 * W]
    h = torch.nn.functional.gelu(y2 @ p["wg"].t(), approximate="tanh") * (y2 @ p["wu"].t())
    x3 = x2 + p["mod"][:, 2 * W:] * (h @ p["wd"].t())
    y3 = unit(x3) * (1 + p["gamma2"])
    g = torch.autograd.grad((y3 * torch.from_numpy(d_y)).sum() + (x3 * torch.from_numpy(d_x)).sum(), list(p.values()))
    return {"y": y3.detach(), "x3": x3.detach()}, dict(zip(p, g))


def test_layer_and_its_gradients():
    """32 bits.  Every step of the chain (12 deep) is within (n + 20) u of its sums' magnitudes, n <= 2 * 136 terms, and
    magnitudes exceed the values' largest by a factor below 8: 12 * 8 * 292 * 2^-24 = 1.7e-3 of a tensor's largest value."""
    import torch
    p, d_y, d_x = _parameters()
    out, d = _layer({n: torch.from_numpy(t).cuda() for n, t in p.items()}, torch.from_numpy(d_y).cuda(), torch.from_numpy(d_x).cuda(),
                    torch.float32)
    want_out, want = _reference(p, d_y.astype(np.float64), d_x.astype(np.float64))
    assert set(d) == set(want)
    for got, ref in ((out, want_out), (d, want)):
        for n in ref:
            err = float((got[n].double().cpu().view(ref[n].shape) - ref[n]).abs().max())
            assert err <= 1.7e-3 * float(ref[n].abs().max()), n


def _bf16_inputs(seed):
    """A layer's operands between its linear layers, in bf16 on a 32-bit stream; sizes with partial sums in every call."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    b = lambda *s: n(*s).bfloat16()  # noqa: E731
    return dict(x=n(300, 256), f=b(300, 256), post=0.1 * n(256), alpha=n(1), gate=n(3, 256), scale=n(256), dy=b(300, 256), d_out=n(300, 256),
                q=b(2, 40, 8, 64), k=b(2, 300, 2, 64), v=b(2, 300, 2, 64), k_len=torch.tensor([300, 130], dtype=torch.int32, device="cuda"),
                dout=b(2, 40, 8, 64), k2=b(2, 12, 2, 64), v2=b(2, 12, 2, 64), wg=0.1 * b(512, 256), wu=0.1 * b(512, 256), xm=b(70, 256),
                dh=b(70, 512))


def _all_calls(t, stream=None):
    from paper_2609_34170_amd import ravel
    import torch
    res = {}
    mod = dict(f=t["f"], post=t["post"], alpha=t["alpha"], gate=t["gate"], scale=t["scale"], group=100)
    res["y"], res["x_out"] = ravel.norm_residual(t["x"], **mod, stream=stream)
    res.update({"d" + k: v for k, v in ravel.norm_residual_grad(res["x_out"], t["dy"], t["d_out"], **mod, stream=stream).items()})
    lens = {"k_len": t["k_len"]}
    for i, (k, v, kw) in enumerate(((t["k"], t["v"], lens), (t["k2"], t["v2"], {}))):
        lse = torch.empty((2, 8, 40), device="cuda")
        o = ravel.cross_attention(t["q"], k, v, lse=lse, **kw, stream=stream)
        g = ravel.cross_attention_grad(t["q"], k, v, o, lse, t["dout"], **kw, stream=stream)
        res.update({f"o{i}": o, f"lse{i}": lse, f"dq{i}": g[0], f"dk{i}": g[1], f"dv{i}": g[2]})
    one = torch.empty((2, 8, 1), device="cuda")
    res["token"] = ravel.cross_attention(t["q"][:, :1], t["k"], t["v"], lse=one, **lens, stream=stream)
    gate, up = (torch.empty((70, 512), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    res["h"] = ravel.gated_mlp(t["xm"], t["wg"], t["wu"], gate=gate, up=up, stream=stream)
    res["h1"] = ravel.gated_mlp(t["xm"][:1], t["wg"], t["wu"], stream=stream)
    res["dxm"], res["dwg"], res["dwu"] = ravel.gated_mlp_grad(t["xm"], t["wg"], t["wu"], gate, up, t["dh"], stream=stream)
    return res


def _copy(t):
    return {k: v.clone() for k, v in t.items()}


def _equal(a, b):
    return [k for k in a if not (a[k] == b[k]).all()]


def test_captured_calls_replay_like_eager_ones():
    """Two graphs of all calls with memory of their own, replayed in turn and side by side with new inputs, with eager calls
    and synchronizations between the replays."""
    import torch
    static = [_bf16_inputs(s) for s in (1, 2)]
    for t in static:
        _all_calls(t)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for t in static:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_all_calls(t))
        graphs.append(g)
    side = [torch.cuda.Stream() for _ in graphs]
    for turn in range(3):
        fresh = [_bf16_inputs(10 * turn + s) for s in (3, 4)]
        want = [_copy(_all_calls(t)) for t in fresh]
        for t, new in zip(static, fresh):
            for k in t:
                t[k].copy_(new[k])
        torch.cuda.synchronize()
        if turn == 1:  # at once
            for s, g in zip(side, graphs):
                with torch.cuda.stream(s):
                    g.replay()
        else:
            for g in graphs:
                g.replay()
        again = _all_calls(fresh[0])  # eager work beside the replays
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert not _equal(o, w), (turn, _equal(o, w))
        assert not _equal(again, want[0])


def test_streams_of_the_callers_choice():
    import torch
    t = _bf16_inputs(7)
    want = _copy(_all_calls(t))
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got_a, got_b = _all_calls(t, stream=a), _all_calls(t, stream=b.cuda_stream)  # two calls at once
    with torch.cuda.stream(a):
        got_c = _all_calls(t)
    torch.cuda.synchronize()
    for got in (got_a, got_b, got_c):
        assert not _equal(got, want)


def test_the_binding_refuses():
    import torch
    from paper_2609_34170_amd import ravel
    t = _bf16_inputs(9)
    x, f, q, k, v, wg, wu, xm = (t[n] for n in ("x", "f", "q", "k", "v", "wg", "wu", "xm"))
    lse = torch.empty((2, 8, 40), device="cuda")
    out = ravel.cross_attention(q, k, v, lse=lse)
    gate, up = torch.empty((70, 512), device="cuda").bfloat16(), torch.empty((70, 512), device="cuda").bfloat16()
    bad = [
        lambda: ravel.norm_residual(x[0]), lambda: ravel.norm_residual(x.double(), f), lambda: ravel.norm_residual(x, f[:, :128]),
        lambda: ravel.norm_residual(x, f.t()), lambda: ravel.norm_residual(x, f, post=t["post"].bfloat16()),
        lambda: ravel.norm_residual(x, f, gate=t["gate"][:, ::2]), lambda: ravel.norm_residual(x, f, gate=t["gate"], scale=t["x"]),
        lambda: ravel.norm_residual(x, f, gate=t["gate"][:1].expand(3, 256)), lambda: ravel.norm_residual(x, x_out=x.clone()),
        lambda: ravel.norm_residual(x, f, alpha=t["post"]), lambda: ravel.norm_residual(x, f, y=torch.empty_like(x)),
        lambda: ravel.norm_residual(x, f.cpu()), lambda: ravel.norm_residual_grad(x, t["dy"], t["d_out"], grads={"gate": None}),
        lambda: ravel.norm_residual_grad(x, t["dy"], f), lambda: ravel.norm_residual_grad(x, t["dy"], scale=t["scale"], grads={"scale": t["gate"]}),
        lambda: ravel.cross_attention(q, k, v.float()), lambda: ravel.cross_attention(q, k[:1], v[:1]),
        lambda: ravel.cross_attention(q, k, v, k_len=t["k_len"].long()), lambda: ravel.cross_attention(q, k, v, q_len=t["k_len"][:1]),
        lambda: ravel.cross_attention(q, k, v, lse=lse[:, :, :1]), lambda: ravel.cross_attention(q.half(), k.half(), v.half()),
        lambda: ravel.cross_attention(q, k.transpose(2, 3).contiguous().transpose(2, 3), v),
        lambda: ravel.cross_attention_grad(q, k, v, out, lse.bfloat16(), t["dout"]),
        lambda: ravel.cross_attention_grad(q, k, v, out[:, :1], lse, t["dout"]),
        lambda: ravel.gated_mlp(xm, wg, wu, act="relu"), lambda: ravel.gated_mlp(xm, wg, wu[:8]), lambda: ravel.gated_mlp(xm.float(), wg, wu),
        lambda: ravel.gated_mlp(xm, wg, wu, gate=gate), lambda: ravel.gated_mlp(xm[:, :128], wg, wu), lambda: ravel.gated_mlp(xm, wg.t(), wu.t()),
        lambda: ravel.gated_mlp_grad(xm, wg, wu, gate, up, t["dh"].float()), lambda: ravel.gated_mlp_grad(xm, wg, wu, None, None, t["dh"], dwg=wg),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((ValueError, ravel.RavelError)):
            call()
            raise AssertionError(i)
    with pytest.raises(ravel.RavelError, match="E_SHAPE"):
        ravel.norm_residual(torch.zeros((2, 12), device="cuda"))
    with pytest.raises(ravel.RavelError, match="E_INVALID"):
        ravel.gated_mlp(xm, wg, wu, h=torch.empty((70, 512), device="cuda").bfloat16(), gate=gate, up=gate)
    with pytest.raises(ravel.RavelError, match="E_INVALID"):
        ravel.cross_attention_grad(q, k, v, out, lse, t["dout"], dk=k)
