"""A key that is minus infinity in one place has a probability of 0 in every row that sees it: nothing but the queries'
gradients at that place (0 times infinity) may differ from a call without the key."""

import pytest

from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,B,R,K,q_len", [
    ((8, 2, 64), 2, 12, 20, None), ((8, 2, 64), 2, 12, 40, None), ((8, 2, 64), 2, 13, 100, [13, 5]), ((4, 4, 32), 1, 1, 7, None),
    ((4, 4, 32), 1, 3, 70, None), ((8, 1, 256), 2, 50, 16, [50, 0]), ((8, 1, 256), 2, 9, 33, [1, 9]), ((8, 4, 128), 64, 33, 100, None),
    ((16, 4, 64), 64, 33, 300, None), ((10, 2, 128), 1, 27, 31, [26])])
def test_a_key_that_no_row_takes(dtype, heads, B, R, K, q_len):
    import torch
    from paper_2609_34170_amd import ravel
    nq, nkv, hd = heads
    T = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator(device="cuda").manual_seed(R + K)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    q, k, v, dout = (n(B, R, nq, hd).abs() + 0.1).to(T), n(B, K, nkv, hd).to(T), n(B, K, nkv, hd).to(T), n(B, R, nq, hd).to(T)
    k[:, K - 1, :, 5] = -float("inf")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    ql = None if q_len is None else ints(q_len)
    res = []
    for kl in (None, ints([K - 1] * B)):
        lse = torch.empty((B, nq, R), device="cuda")
        out = ravel.cross_attention(q, k, v, ql, kl, lse=lse)
        res.append((out, lse, *ravel.cross_attention_grad(q, k, v, out, lse, dout, ql, kl)))
    (out, lse, dq, dk, dv), (out1, lse1, dq1, dk1, dv1) = res
    assert torch.equal(out, out1) and torch.equal(lse, lse1)
    assert torch.equal(dv, dv1) and not bool(dv[:, K - 1].any())
    assert torch.equal(dk, dk1) and not bool(dk[:, K - 1].any())
    rest = [i for i in range(hd) if i != 5]
    assert torch.equal(dq[..., rest], dq1[..., rest])
