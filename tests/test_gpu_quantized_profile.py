"""ravel_profile_step on buffers with 8-bit contexts: a record a launch, with the bytes and operations of the tokens that
are there."""

import pytest

import synth
from tests.harness import have_gpu
from tests.test_gpu_quantized_context import Roll

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("name,kw,joined", [("pi_b1", dict(layers=2, prefix_len=816), True),
                                            ("small_bf16", dict(layers=3, prefix_len=100, batch=2), False),
                                            ("tiny_fp32", dict(prefix_len=40), False)])
def test_records(name, kw, joined):
    s = synth.get_config(name).replace(**kw)
    g = Roll(s, synth.draw_weights(s, seed=0), s.batch, 0, 32)
    z = synth.draw_fop_tokens(s, 0, 0, batch=s.batch)
    for e in range(s.batch):
        g.set_context(e, *synth.draw_context(s, 2, e, 0), 0)
    g.step(z)
    elt = 2 if s.dtype == synth.workloads.BF16 else 4
    tokens = [s.prefix_len] * s.batch

    def check(track):
        g.buf.track_context(track)
        recs = g.buf.profile_step(g.fop, g.action)
        of = {x: [r for r in recs if r[0] == x] for x in ("cache_attn", "cache_join", "cache_weight")}
        assert [len(of[x]) for x in of] == [s.layers, s.layers * joined, s.layers * track]
        n, H, row = sum(tokens), s.horizon, s.n_kv_heads * s.head_dim
        for _, nbytes, flops, ms in of["cache_attn"]:
            assert flops == 4.0 * s.n_q_heads * s.head_dim * H * (n + s.batch * H)
            assert nbytes >= 2 * n * row + 2 * s.batch * H * (row + s.n_q_heads * s.head_dim) * elt
            assert nbytes < 1.3 * (2 * n * row + 2 * s.batch * H * (row + s.n_q_heads * s.head_dim) * elt)
            assert ms > 0
        for _, nbytes, flops, ms in of["cache_join"]:
            assert nbytes > 0 and ms > 0
        for _, nbytes, flops, ms in of["cache_weight"]:
            assert flops == 2.0 * s.n_q_heads * s.head_dim * H * n
            assert nbytes >= n * row + 8 * n * s.n_kv_heads and ms > 0

    check(False)
    check(True)
    g.buf.evict_context(0, 20, first=1)
    tokens[0] = 20
    check(True)
    check(False)
