"""Inputs whose rows share memory (one row repeated by a stride of 0, windows that overlap): what lies behind a length is masked by its
index, also where its memory is a live row's that holds infinities."""

import pytest

from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]

SIZES = [((8, 2, 64), 2, 3, 20), ((8, 2, 64), 2, 3, 70), ((4, 4, 32), 1, 1, 100), ((8, 1, 256), 2, 9, 33), ((16, 4, 128), 16, 100, 300)]


def _type(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,B,R,K", SIZES)
def test_one_value_for_all_keys(heads, B, R, K, dtype):
    import torch
    from paper_2609_34170_amd import ravel
    nq, nkv, hd = heads
    T = _type(dtype)
    q, k, v = torch.randn(B, R, nq, hd, device="cuda").to(T), torch.randn(B, K, nkv, hd, device="cuda").to(T), torch.zeros(B, 1, nkv, hd, device="cuda").to(T)
    v[..., 3], v[..., 5] = 2, float("inf")
    lens = torch.tensor([K - 1, K] * B, dtype=torch.int32, device="cuda")[:B]
    out = ravel.cross_attention(q, k, v.expand(B, K, nkv, hd), k_len=lens)
    assert bool((out[..., 5] == float("inf")).all())
    # probabilities of at most 300 keys, each rounded once (bf16), summed and normed: 2 within 2^-7
    assert bool(((out[..., 3].float() - 2).abs() <= 2.0 ** -6).all())
    rest = [i for i in range(hd) if i not in (3, 5)]
    assert not bool(out[..., rest].any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,B,R,K", SIZES)
def test_keys_that_overlap(heads, B, R, K, dtype):
    """Key i is half of key i - 1 and half of key i + 1.  The last live key is minus infinity in its second half's first place, which
    takes it out of every row; the first masked one has it in front, where the queries are negative."""
    import torch
    from paper_2609_34170_amd import ravel
    nq, nkv, hd = heads
    T, h = _type(dtype), hd // 2
    q, v = torch.randn(B, R, nq, hd, device="cuda"), torch.randn(B, K, nkv, hd, device="cuda").to(T)
    q[..., 0], q[..., h] = -1, 1
    q, dout = q.to(T), torch.randn(B, R, nq, hd, device="cuda").to(T)
    n = K - 2  # live keys
    line = torch.randn(B, nkv, (K + 1) * h, device="cuda").to(T)
    line[..., n * h] = -float("inf")
    k = line.as_strided((B, K, nkv, hd), (nkv * (K + 1) * h, h, (K + 1) * h, 1))
    res = []
    for live, keys in ((n, k), (n - 1, k.contiguous())):
        lens = torch.full((B,), live, dtype=torch.int32, device="cuda")
        lse = torch.empty(B, nq, R, device="cuda")
        out = ravel.cross_attention(q, keys, v, k_len=lens, lse=lse)
        res.append((out, lse, *ravel.cross_attention_grad(q, keys, v, out, lse, dout, k_len=lens)))
    rest = [i for i in range(hd) if i != h]  # (0 times infinity there)
    for i, (a, b) in enumerate(zip(*res)):
        assert torch.equal(a[..., rest], b[..., rest]) if i == 2 else torch.equal(a, b), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,F", [(70, 72, 40), (200, 264, 520), (1, 72, 40), (3, 1032, 520)])
def test_one_input_row_for_all(M, K, F, dtype):
    import torch
    from paper_2609_34170_amd import ravel
    T = _type(dtype)
    n = lambda *s: torch.randn(*s, device="cuda").to(T)  # noqa: E731
    x, wg, wu = n(1, K), n(F, K), n(F, K)
    gate, up, dh = (torch.ones(M, F, device="cuda", dtype=T) for _ in range(3))
    want = ravel.gated_mlp_grad(x.expand(M, K).contiguous(), wg, wu, gate, up, dh, need_x=False)
    x[0, 3] = float("inf")
    got = ravel.gated_mlp_grad(x.expand(M, K), wg, wu, gate, up, dh, need_x=False)
    for a, b in zip(got[1:], want[1:]):
        assert bool((a[:, 3] == float("inf")).all())
        assert torch.equal(a[:, :3], b[:, :3]) and torch.equal(a[:, 4:], b[:, 4:])
