"""The gated MLP with its gradients on the GPU against the 64-bit definition (tests/layer_oracle.py has the bounds)."""

import numpy as np
import pytest

from tests import layer_oracle as lo
from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


def _dev(x, dtype, pad=0):
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


def _clean(t):
    return bool((t._base[-1] == 7).all()) and bool((t._base[:, t.shape[1]:] == 7).all())


def _near(got, want, tol, name):
    got = got.detach().float().cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])


@pytest.mark.parametrize("dtype,kind,M,K,F,pad,wide", [
    ("bf16", "gelu", 1, 128, 512, 0, False), ("bf16", "silu", 1, 1024, 64, 0, True), ("bf16", "gelu", 3, 8, 8, 8, False),
    ("f32", "silu", 1, 64, 40, 0, False), ("bf16", "gelu", 16, 200, 88, 0, False), ("bf16", "silu", 17, 328, 136, 8, False),
    ("bf16", "gelu", 50, 512, 256, 0, True), ("f32", "gelu", 50, 128, 200, 4, False), ("bf16", "gelu", 64, 72, 1000, 0, False),
    ("bf16", "silu", 65, 1000, 136, 0, False), ("bf16", "gelu", 200, 264, 520, 16, True), ("f32", "silu", 77, 328, 888, 0, False),
    ("bf16", "gelu", 700, 256, 1032, 0, False), ("bf16", "silu", 1111, 136, 2056, 0, False), ("f32", "gelu", 300, 72, 264, 0, False),
    ("bf16", "gelu", 2100, 520, 4096, 0, False), ("bf16", "silu", 4200, 264, 4096, 8, False),  # the last: rows in two pieces
    ("f32", "gelu", 513, 1032, 520, 0, False),
    # every tile of the gradients' products, whole and in ranges of the contraction
    ("bf16", "gelu", 70, 72, 8200, 0, False), ("bf16", "silu", 70, 1544, 2568, 8, False), ("bf16", "gelu", 70, 1544, 2568, 0, True),
    ("bf16", "gelu", 777, 2568, 72, 0, False), ("bf16", "silu", 2100, 4104, 72, 8, False), ("bf16", "silu", 3000, 72, 4104, 0, False),
    ("bf16", "gelu", 4200, 136, 6152, 8, True), ("bf16", "silu", 4200, 136, 6152, 0, False), ("f32", "gelu", 70, 1032, 1544, 4, False),
    ("f32", "silu", 520, 72, 4104, 0, False), ("f32", "gelu", 3000, 1032, 72, 0, False), ("f32", "silu", 70, 4104, 520, 0, False)])
def test_forward_and_gradients(dtype, kind, M, K, F, pad, wide):
    import torch
    from paper_2609_34170_amd import ravel
    r = np.random.default_rng(M + K + F)
    n = lambda s, *shape: lo.held(s * r.standard_normal(shape), dtype)  # noqa: E731
    x, wg, wu, dh = n(1, M, K), n(2 / K ** 0.5, F, K), n(1 / K ** 0.5, F, K), n(1, M, F)
    t = [_dev(v, dtype, pad) for v in (x, wg, wu)]
    h, gate, up = (_out(M, F, dtype, pad) for _ in range(3))
    ravel.gated_mlp(*t, act=kind, h=h, gate=gate, up=up)
    torch.cuda.synchronize()
    want, tol = lo.mlp(x, wg, wu, kind, dtype)
    for name, v in (("gate", gate), ("up", up), ("h", h)):
        _near(v, want[name], tol[name], name)
        assert _clean(v), name
    assert torch.equal(ravel.gated_mlp(*t, act=kind), h)  # without gate and up

    W = "f32" if wide else dtype
    dx, dwg, dwu = _out(M, K, dtype, pad), _out(F, K, W, pad), _out(F, K, W, pad)
    ravel.gated_mlp_grad(*t, gate, up, _dev(dh, dtype, pad), act=kind, dx=dx, dwg=dwg, dwu=dwu)
    torch.cuda.synchronize()
    want, tol = lo.mlp_grad(x, wg, wu, gate.double().cpu().numpy(), up.double().cpu().numpy(), dh, kind, dtype, W)
    for name, v in (("dx", dx), ("dwg", dwg), ("dwu", dwu)):
        _near(v, want[name], tol[name], name)
        assert _clean(v), name
    # one at a time, and the same bits again
    one = ravel.gated_mlp_grad(*t, gate, up, _dev(dh, dtype), act=kind, need_w=False)
    assert torch.equal(one[0], dx) and one[1] is None and one[2] is None
    one = ravel.gated_mlp_grad(*t, gate, up, _dev(dh, dtype), act=kind, need_x=False, weight_dtype=dwg.dtype)
    assert one[0] is None and torch.equal(one[1], dwg) and torch.equal(one[2], dwu)


def test_no_rows():
    import torch
    from paper_2609_34170_amd import ravel
    x, w = torch.empty((0, 64), device="cuda").bfloat16(), torch.randn((32, 64), device="cuda").bfloat16()
    h = ravel.gated_mlp(x, w, w.clone())
    assert h.shape == (0, 32)
    dx, dwg, dwu = ravel.gated_mlp_grad(x, w, w.clone(), h, h.clone(), h.clone())
    assert dx.shape == (0, 64) and (dwg == 0).all() and (dwu == 0).all()


@pytest.mark.parametrize("kind", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_activations_far_out(kind, dtype):
    """Gate values up to the largest numbers: the activation goes to x and to 0, its slope to 1 and to 0.  (Below 2^-60 of
    the gate value either is as good as 0.)"""
    import torch
    from paper_2609_34170_amd import ravel
    a = np.concatenate([np.linspace(-3e4, 3e4, 41), np.linspace(-12, 12, 81), [1e15, -1e15, 3e38, -3e38, 0.0, 1e-30, -1e-30]])
    a = lo.held(np.concatenate([a, np.zeros(136 - len(a))]), dtype)
    x, wg, wu = np.eye(136), np.diag(a), np.ones((136, 136))
    t = [_dev(v, dtype) for v in (x, wg, wu)]
    gate, up = (torch.empty((136, 136), dtype=t[0].dtype, device="cuda") for _ in range(2))
    h = ravel.gated_mlp(*t, act=kind, gate=gate, up=up)
    dx, dwg, dwu = ravel.gated_mlp_grad(*t, gate, up, torch.ones_like(h), act=kind)
    far, b = np.abs(a) > 60, np.clip(a, -60, 60)
    want, slope = lo.act(b, kind)
    want, slope = np.where(far, np.maximum(a, 0), want), np.where(far, (a > 0) * 1.0, slope)
    got, got_slope = (torch.diagonal(v).double().cpu().numpy() for v in (h, dwg))  # dwg[i, i] = dh up slope(a_i)
    assert (np.abs(got - want) <= (lo.ACT + 2 * lo.H[dtype]) * np.abs(want) + 2.0 ** -60 * np.abs(a)).all()
    assert (np.abs(got_slope - slope) <= 2 * lo.ACT * (1 + np.abs(b)) + 2 * lo.H[dtype] * np.abs(slope)).all()


def test_values_that_are_not_finite_stay_in_their_row():
    import torch
    from paper_2609_34170_amd import ravel
    r = torch.randn
    x, wg, wu = r((70, 72), device="cuda").bfloat16(), r((40, 72), device="cuda").bfloat16(), r((40, 72), device="cuda").bfloat16()
    h0 = ravel.gated_mlp(x, wg, wu)
    x[69, 71] = float("nan")
    h = ravel.gated_mlp(x, wg, wu)
    assert torch.isnan(h[69].float()).all() and torch.equal(h[:69], h0[:69])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_single_row_has_no_stride(dtype):
    """As far as dwg = dg x is infinite where x is, and nothing else."""
    import torch
    from paper_2609_34170_amd import ravel
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    n = lambda *s: torch.randn(*s, device="cuda").to(t)  # noqa: E731
    x, wg, wu, dh, gate, up = n(1, 72), n(40, 72), n(40, 72), n(1, 40), n(1, 40), n(1, 40)
    x[0, 3] = float("inf")
    odd = x.as_strided((1, 72), (0, 1))
    got = [ravel.gated_mlp_grad(a, wg, wu, gate, up, dh) for a in (x, odd)]
    for one, other in zip(*got):
        assert torch.equal(one, other)
    assert torch.isinf(got[1][1][:, 3].float()).all() and torch.isfinite(got[1][1][:, 4:].float()).all()
