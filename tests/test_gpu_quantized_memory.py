"""The device memory that a buffer with 8-bit contexts takes."""

import pytest

import synth
from tests.harness import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


def _used(make):
    import torch
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    x = make()
    torch.cuda.synchronize()
    return before - torch.cuda.mem_get_info()[0], x


@pytest.mark.parametrize("dtype,layers,heads", [("bf16", 8, (8, 1, 256)), ("f32", 8, (8, 8, 64))])
def test_one_env_takes_about_half_the_memory(dtype, layers, heads):
    """Of a context of N key elements and as many values, two slots: bf16 8 N bytes, 32 bits 16 N; codes 4 N, scales,
    weights and eviction's indices (16 / head_dim + 16 / (block head_dim)) N.  Contexts in host memory take 2 N elements
    more, from the first of them on."""
    import torch
    from paper_2609_34170_amd import ravel
    nq, nkv, hd = heads
    s = synth.get_config("small_bf16" if dtype == "bf16" else "tiny_fp32").replace(
        layers=layers, n_q_heads=nq, n_kv_heads=nkv, head_dim=hd, prefix_len=16384 // nkv * 256 // hd)
    elt = 2 if dtype == "bf16" else 4
    n = layers * s.prefix_len * nkv * hd
    model = ravel.Model(s, synth.draw_weights(s, seed=0))
    for block in (0, 64):  # what a model's first buffers set up
        ravel.Buffer(model, 1, 0, quantized=block).close()
    plain, p = _used(lambda: ravel.Buffer(model, 1, 0))
    p.close()
    quant, q = _used(lambda: ravel.Buffer(model, 1, 0, quantized=64))
    least = 4 * n + (16 / hd + 16 / (64 * hd)) * n
    slack = 0.03 * 4 * n * elt  # a buffer's attention workspace differs; allocations come in steps of 2 MiB
    assert plain >= 4 * n * elt, (plain, n)
    assert quant - (plain - 4 * n * elt) <= least + slack, (plain, quant, n)
    T = torch.bfloat16 if dtype == "bf16" else torch.float32
    shape = (layers, s.prefix_len, nkv, hd)
    k = torch.ones(shape, dtype=T, device="cuda")
    host = torch.ones(shape, dtype=T, pin_memory=True)
    assert _used(lambda: q.set_context(0, k, k, 0))[0] <= slack
    assert abs(_used(lambda: q.set_context(0, host, host, 0))[0] - 2 * n * elt) <= slack
    assert _used(lambda: q.set_context(0, host, k, 0))[0] <= slack
    q.close()
