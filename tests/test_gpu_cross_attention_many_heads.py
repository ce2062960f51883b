"""Cross attention with as many heads and as few rows as one launch holds, and with rows that end anywhere in a tile."""

import numpy as np
import pytest

from tests import layer_oracle as lo
from tests.harness import have_gpu
from tests.test_gpu_cross_attention import _case, _compare, _near, _run

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("batch,heads,need_kv", [(32768, 64, True), (65535, 256, False)])
def test_one_row_of_millions_of_heads(batch, heads, need_kv):
    """33 keys of 32 dims, shared by all batch rows; batch rows at both ends and between against the definition."""
    import torch
    from paper_2609_34170_amd import ravel
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *s: torch.randn(s, generator=g, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    q, dout, k, v = n(batch, 1, heads, 32), n(batch, 1, heads, 32), n(1, 33, heads, 32), n(1, 33, heads, 32)
    kb, vb = (t.expand(batch, 33, heads, 32) for t in (k, v))
    lse = torch.empty((batch, heads, 1), device="cuda")
    out = ravel.cross_attention(q, kb, vb, lse=lse)
    dq, dk, dv = ravel.cross_attention_grad(q, kb, vb, out, lse, dout, need_kv=need_kv)
    at = [0, 1, batch // 2, batch - 1]
    host = lambda t: t[at].double().cpu().numpy()  # noqa: E731
    want, tol = lo.attention(host(q), host(kb), host(vb), dout=host(dout))
    for name, got in (("out", out), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        if got is not None:
            _near(got[at], want[name], tol[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,R,K", [((4, 4, 32), 1, 33), ((8, 1, 64), 2, 40), ((6, 2, 128), 5, 33), ((4, 2, 256), 9, 64),
                                       ((4, 4, 64), 63, 100), ((4, 4, 128), 65, 70), ((2, 1, 32), 65, 300)])
def test_rows_that_end_inside_a_tile(dtype, heads, R, K):
    """Statistics of rows behind the last are none's; the workspace that they would lie in holds NaN."""
    import torch
    c = _case(dtype, heads, 3, R, K, [R, 0, max(R - 1, 1)], [K, K - 1, 1])
    c["q_len"][1] = R // 2
    junk = torch.full((1 << 22,), float("nan"), device="cuda")  # (the calls' workspaces come from here)
    del junk
    _, _, got = _run(c)
    _compare(c, got)
