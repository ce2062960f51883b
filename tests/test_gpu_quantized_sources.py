"""Where buffers with 8-bit contexts take them from: host or device memory, at any alignment."""

import numpy as np
import pytest

import synth
from tests.harness import have_gpu
from tests.test_gpu_quantized_context import _quantised

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="needs a GPU")]


@pytest.mark.parametrize("name,kw,block", [("small_bf16", dict(layers=3, prefix_len=77), 16),
                                           ("tiny_fp32", dict(layers=2), 32)])
def test_contexts_from_anywhere(name, kw, block):
    """Host memory, pinned or not, and device memory, at any alignment of an element: the same codes; one after the other
    on several streams."""
    import torch
    from paper_2609_34170_amd import ravel
    s = synth.get_config(name).replace(batch=1, **kw)
    model = ravel.Model(s, synth.draw_weights(s, seed=0))
    b = ravel.Buffer(model, 1, 0, quantized=block)
    b.set_option(ravel.OPT_SYNC_CONTEXT, 1)
    T = torch.bfloat16 if s.dtype == synth.workloads.BF16 else torch.float32
    action = torch.empty((1, s.action_dim), device="cuda")
    fop = torch.zeros((1, s.n_fop, s.width), dtype=T, device="cuda") if s.n_fop else None

    def place(x, where, shift):
        x = torch.from_numpy(np.ascontiguousarray(x)).to(T)
        room = torch.empty(x.numel() + 64, dtype=T, pin_memory=where == "pinned", device="cuda" if where == "cuda" else "cpu")
        at = next(i for i in range(64) if room[i:].data_ptr() % 64 == 0) + shift
        room[at:at + x.numel()] = x.flatten().to(room.device)
        return room[at:at + x.numel()].view(x.shape)

    streams, t, keep = [torch.cuda.Stream() for _ in range(3)], 0, []
    for where in ("cuda", "cpu", "pinned"):
        for shifts in ((0, 0), (1, 0), (0, 3), (1, 1)):
            k, v = synth.draw_context(s, 9, 0, t)
            kd, vd = place(k, where, shifts[0]), place(v, where, shifts[1])
            keep.append((kd, vd))
            torch.cuda.synchronize()
            b.set_context(0, kd, vd, t, stream=streams[t % 3])
            b.step(fop, action)
            torch.cuda.synchronize()
            want, _ = _quantised(k, v, block)
            c = b.context_cache(0)
            assert torch.equal(c.k.cpu(), torch.from_numpy(want["k"])), (where, shifts)
            assert torch.equal(c.v.cpu(), torch.from_numpy(want["v"])), (where, shifts)
            assert torch.equal(c.k_scale.cpu(), torch.from_numpy(want["ks"])), (where, shifts)
            assert c.length.tolist() == [s.prefix_len] * s.layers
            t += 1


def test_contexts_in_host_memory_one_behind_the_other():
    """Several envs' contexts in one call and in calls without a wait between them share the way in."""
    import torch
    from paper_2609_34170_amd import ravel
    s = synth.get_config("small_bf16").replace(layers=4, batch=3, prefix_len=301)
    model = ravel.Model(s, synth.draw_weights(s, seed=0))
    b = ravel.Buffer(model, 3, 0, quantized=64)
    b.set_option(ravel.OPT_SYNC_CONTEXT, 1)
    ks, vs = zip(*(synth.draw_context(s, 2, e, 0) for e in range(3)))
    pin = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).pin_memory()  # noqa: E731
    k, v = pin(np.stack(ks)), pin(np.stack(vs))
    k2, v2 = pin(ks[2][:, ::-1]), pin(vs[2][:, ::-1])
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    b.set_context(-1, k, v, 0, stream=streams[0])
    b.set_context(0, k[1], v[1], 1, stream=streams[0])
    streams[1].wait_stream(streams[0])  # env 0's and 2's slots are written once more
    b.set_context(2, k2, v2, 1, stream=streams[1])
    b.set_context(1, k[0], v[0], 1, stream=streams[1])
    action = torch.empty((3, s.action_dim), device="cuda")
    fop = torch.zeros((3, s.n_fop, s.width), dtype=torch.bfloat16, device="cuda")
    b.step(fop, action)
    torch.cuda.synchronize()
    for e, (wk, wv) in enumerate([(ks[1], vs[1]), (ks[0], vs[0]), (ks[2][:, ::-1], vs[2][:, ::-1])]):
        want, _ = _quantised(wk, wv, 64)
        c = b.context_cache(e)
        assert torch.equal(c.k.cpu(), torch.from_numpy(want["k"])), e
        assert torch.equal(c.v.cpu(), torch.from_numpy(want["v"])), e
