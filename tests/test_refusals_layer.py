"""What a layer's operators refuse: every check answers on the host, before anything is launched."""

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_34170_amd", "libravel.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libravel.so not built")

P = 1 << 20  # aligned addresses that are never read
INVALID, SHAPE = -1, -4


def _ravel():
    from paper_2609_34170_amd import ravel
    ravel.load_library()
    return ravel


def _addr(i):
    return P * (i + 1)


def _norm(**kw):
    d = dict(stream_dtype=0, dtype=1, rows=10, width=64, mods=10, group=1, eps=1e-6, reserved=0, x=_addr(0), f=_addr(1),
             post=_addr(2), alpha=_addr(3), gate=_addr(4), scale=_addr(5), shift=_addr(6), x_out=_addr(7), y=_addr(8),
             x_stride=64, f_stride=64, x_out_stride=64, y_stride=64, gate_stride=64, scale_stride=192, shift_stride=192)
    d.update(kw)
    return _ravel().RavelNorm(**d)


def _norm_grad(**kw):
    d = dict(dy=_addr(9), d_out=_addr(10), dx=_addr(11), df=_addr(12), dpost=_addr(13), dalpha=_addr(14), dgate=_addr(15),
             dscale=_addr(16), dshift=_addr(17), dy_stride=64, d_out_stride=64, dx_stride=64, df_stride=64, dgate_stride=64,
             dscale_stride=64, dshift_stride=64, workspace=_addr(40), workspace_bytes=1 << 30)
    d.update(kw)
    return _ravel().RavelNormGrad(**d)


def _cross(**kw):
    s = (4096, 256, 64)
    d = dict(dtype=1, batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, rows=16, keys=16, scale=0.125, q_len=None, k_len=None,
             q=_addr(0), k=_addr(1), v=_addr(2), out=_addr(3), lse=_addr(4), q_stride=s, k_stride=s, v_stride=s, out_stride=s,
             workspace=_addr(40), workspace_bytes=1 << 30)
    d.update(kw)
    return _ravel().RavelCross(**d)


def _cross_grad(**kw):
    s = (4096, 256, 64)
    d = dict(dout=_addr(5), dq=_addr(6), dk=_addr(7), dv=_addr(8), dout_stride=s, dq_stride=s, dk_stride=s, dv_stride=s,
             workspace=_addr(40), workspace_bytes=1 << 30)
    d.update(kw)
    return _ravel().RavelCrossGrad(**d)


def _mlp(**kw):
    d = dict(dtype=1, act=0, rows=10, width=64, hidden=128, reserved=0, x=_addr(0), wg=_addr(1), wu=_addr(2), h=_addr(3),
             gate=_addr(4), up=_addr(5), x_stride=64, w_stride=64, h_stride=128, gate_stride=128, workspace=_addr(40),
             workspace_bytes=1 << 30)
    d.update(kw)
    return _ravel().RavelMlp(**d)


def _mlp_grad(**kw):
    d = dict(weight_dtype=1, reserved=0, dh=_addr(6), dx=_addr(7), dwg=_addr(8), dwu=_addr(9), dh_stride=128, dx_stride=64,
             dw_stride=64, workspace=_addr(40), workspace_bytes=1 << 30)
    d.update(kw)
    return _ravel().RavelMlpGrad(**d)


def _call(name, *structs):
    lib = _ravel().load_library()
    return getattr(lib, name)(*[None if s is None else ctypes.byref(s) for s in structs], None)


def _refused(status, want):
    assert status == want
    assert _ravel().load_library().ravel_last_error()


BOTH_NORM = [(dict(stream_dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(stream_dtype=1, dtype=0), INVALID),
             (dict(rows=-1), SHAPE), (dict(width=0), SHAPE), (dict(width=68), SHAPE), (dict(width=8200), SHAPE),
             (dict(rows=1 << 23), SHAPE), (dict(mods=0), SHAPE), (dict(group=0), SHAPE), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
             (dict(eps=float("inf")), INVALID), (dict(reserved=1), INVALID), (dict(f=_addr(1) + 8), INVALID),
             (dict(gate=_addr(4) + 4), INVALID), (dict(alpha=_addr(3) + 2), INVALID), (dict(f_stride=66), SHAPE),
             (dict(f_stride=-64), SHAPE), (dict(x_out_stride=62), SHAPE), (dict(scale_stride=65), SHAPE),
             (dict(x_out=None), INVALID)]


@pytest.mark.parametrize("kw,status", BOTH_NORM + [
    (dict(x=None), INVALID), (dict(y=_addr(0)), INVALID), (dict(y=_addr(1)), INVALID), (dict(x_out=_addr(1)), INVALID),
    (dict(x_out=_addr(8)), INVALID), (dict(y_stride=56), SHAPE), (dict(x_stride=1 << 61), SHAPE),
    (dict(f=None), INVALID), (dict(f=None, post=None, alpha=None, gate=None), INVALID),  # x_out without f
    (dict(f=None, post=None, alpha=None, gate=None, x_out=None, y=None), INVALID),  # nothing to compute
    (dict(x_out=_addr(0), x_stride=128), INVALID)])
def test_norm(kw, status):
    _refused(_call("ravel_norm_residual", _norm(**kw)), status)


@pytest.mark.parametrize("kw,status", BOTH_NORM)
def test_norm_grad_inputs(kw, status):
    _refused(_call("ravel_norm_residual_grad", _norm(**kw), _norm_grad()), status)


@pytest.mark.parametrize("kw,of,status", [
    (dict(), dict(post=None), INVALID), (dict(), dict(alpha=None), INVALID), (dict(), dict(gate=None), INVALID),
    (dict(), dict(scale=None), INVALID), (dict(dx_stride=32), {}, SHAPE), (dict(df_stride=0), {}, SHAPE),
    (dict(dgate_stride=0), {}, SHAPE), (dict(dscale_stride=64), dict(scale_stride=0), SHAPE), (dict(dshift_stride=60), {}, SHAPE),
    (dict(dx=_addr(7)), {}, INVALID), (dict(df=_addr(10)), {}, INVALID), (dict(dgate=_addr(16)), {}, INVALID),
    (dict(dx=_addr(10), d_out_stride=128), {}, INVALID), (dict(dy=_addr(9) + 4), {}, INVALID), (dict(dpost=_addr(13) + 4), {}, INVALID),
    (dict(workspace=None), {}, INVALID), (dict(workspace_bytes=8), {}, INVALID), (dict(workspace_bytes=-1), {}, INVALID),
    (dict(workspace=_addr(40) + 16), {}, INVALID)])
def test_norm_grad(kw, of, status):
    _refused(_call("ravel_norm_residual_grad", _norm(rows=1000, mods=1000, **of), _norm_grad(**kw)), status)


BOTH_CROSS = [(dict(dtype=2), INVALID), (dict(batch=-1), SHAPE), (dict(batch=65536), SHAPE), (dict(n_q_heads=3), SHAPE),
              (dict(n_q_heads=0), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_q_heads=258), SHAPE), (dict(head_dim=96), SHAPE),
              (dict(head_dim=512), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 20) + 1), SHAPE), (dict(keys=-1), SHAPE),
              (dict(keys=(1 << 24) + 1), SHAPE), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
              (dict(scale=2.0 ** 101), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(out=None), INVALID),
              (dict(v=_addr(2) + 8), INVALID), (dict(k_len=_addr(9) + 2), INVALID), (dict(q_stride=(4096, 256, 60)), SHAPE),
              (dict(k_stride=(4096, -256, 64)), SHAPE), (dict(v_stride=(4096, 1 << 22, 64)), SHAPE),
              (dict(q_stride=(1 << 60, 256, 64)), SHAPE),
              (dict(batch=65535, rows=1 << 20), SHAPE)]  # more tiles than a launch holds


@pytest.mark.parametrize("kw,status", BOTH_CROSS + [
    (dict(out=_addr(0)), INVALID), (dict(out=_addr(1)), INVALID), (dict(lse=_addr(3)), INVALID), (dict(lse=_addr(4) + 2), INVALID),
    (dict(out_stride=(4096, 0, 64)), SHAPE), (dict(out_stride=(4096, 256, 32)), SHAPE), (dict(k_len=_addr(3)), INVALID),
    (dict(keys=100000, workspace=None), INVALID), (dict(keys=100000, workspace_bytes=1024), INVALID),
    (dict(keys=100000, workspace=_addr(40) + 128), INVALID)])
def test_cross(kw, status):
    _refused(_call("ravel_cross_attention", _cross(**kw)), status)


@pytest.mark.parametrize("kw,status", BOTH_CROSS + [(dict(lse=None), INVALID), (dict(out_stride=(4096, -8, 64)), SHAPE)])
def test_cross_grad_inputs(kw, status):
    _refused(_call("ravel_cross_attention_grad", _cross(**kw), _cross_grad()), status)


@pytest.mark.parametrize("kw,status", [
    (dict(dk=None), INVALID), (dict(dv=None), INVALID), (dict(dout=None), INVALID), (dict(dq=_addr(0)), INVALID),
    (dict(dv=_addr(7)), INVALID), (dict(dk=_addr(5)), INVALID), (dict(dq_stride=(4096, 0, 64)), SHAPE),
    (dict(dk_stride=(4096, 256, 32)), SHAPE), (dict(dv=_addr(8) + 4), INVALID), (dict(workspace=None), INVALID),
    (dict(workspace_bytes=64), INVALID)])
def test_cross_grad(kw, status):
    _refused(_call("ravel_cross_attention_grad", _cross(keys=200), _cross_grad(**kw)), status)


def test_cross_grad_tiles_of_keys():
    n = ctypes.c_int64(0)
    many = _cross(batch=60000, rows=1, keys=1 << 20)
    name = "ravel_cross_attention_grad_workspace"
    _refused(getattr(_ravel().load_library(), name)(ctypes.byref(many), ctypes.byref(_cross_grad()), ctypes.byref(n)), SHAPE)
    dq = _cross_grad(dk=None, dv=None)
    assert getattr(_ravel().load_library(), name)(ctypes.byref(many), ctypes.byref(dq), ctypes.byref(n)) == 0


BOTH_MLP = [(dict(dtype=2), INVALID), (dict(act=2), INVALID), (dict(rows=-1), SHAPE), (dict(width=60), SHAPE), (dict(width=0), SHAPE),
            (dict(hidden=4), SHAPE), (dict(hidden=(1 << 18) + 8), SHAPE), (dict(reserved=1), INVALID), (dict(x=None), INVALID),
            (dict(wg=None), INVALID), (dict(wu=_addr(2) + 8), INVALID), (dict(x_stride=60), SHAPE), (dict(w_stride=-64), SHAPE),
            (dict(x_stride=1 << 22), SHAPE), (dict(up=None), INVALID), (dict(gate=None), INVALID)]


@pytest.mark.parametrize("kw,status", BOTH_MLP + [
    (dict(h=None), INVALID), (dict(h_stride=120), SHAPE), (dict(gate_stride=64), SHAPE), (dict(h=_addr(0)), INVALID),
    (dict(gate=_addr(5)), INVALID)])
def test_mlp(kw, status):
    _refused(_call("ravel_gated_mlp", _mlp(**kw)), status)


@pytest.mark.parametrize("kw,status", BOTH_MLP)
def test_mlp_grad_inputs(kw, status):
    _refused(_call("ravel_gated_mlp_grad", _mlp(**kw), _mlp_grad()), status)


@pytest.mark.parametrize("kw,status", [
    (dict(weight_dtype=2), INVALID), (dict(reserved=1), INVALID), (dict(dwg=None), INVALID), (dict(dwu=None), INVALID),
    (dict(dh=None), INVALID), (dict(dx=_addr(0)), INVALID), (dict(dwu=_addr(8)), INVALID), (dict(dx_stride=32), SHAPE),
    (dict(dw_stride=56), SHAPE), (dict(dh_stride=129), SHAPE), (dict(workspace=None), INVALID), (dict(workspace_bytes=100), INVALID)])
def test_mlp_grad(kw, status):
    _refused(_call("ravel_gated_mlp_grad", _mlp(), _mlp_grad(**kw)), status)


def test_null_structs():
    for name, structs in (("ravel_norm_residual", [_norm()]), ("ravel_norm_residual_grad", [_norm(), _norm_grad()]),
                          ("ravel_cross_attention", [_cross()]), ("ravel_cross_attention_grad", [_cross(), _cross_grad()]),
                          ("ravel_gated_mlp", [_mlp()]), ("ravel_gated_mlp_grad", [_mlp(), _mlp_grad()])):
        for i in range(len(structs)):
            _refused(_call(name, *[None if j == i else s for j, s in enumerate(structs)]), INVALID)


def test_workspaces():
    lib, n = _ravel().load_library(), ctypes.c_int64(-1)
    r = ctypes.byref
    assert lib.ravel_norm_residual_grad_workspace(r(_norm()), r(_norm_grad(dpost=None, dalpha=None)), r(n)) == 0 and n.value == 0
    assert lib.ravel_norm_residual_grad_workspace(r(_norm(rows=1000)), r(_norm_grad()), r(n)) == 0 and n.value > 0
    assert lib.ravel_cross_attention_workspace(r(_cross()), r(n)) == 0 and n.value == 0
    assert lib.ravel_cross_attention_workspace(r(_cross(keys=100000)), r(n)) == 0 and n.value > 0
    assert lib.ravel_cross_attention_grad_workspace(r(_cross(rows=0)), r(_cross_grad()), r(n)) == 0
    assert lib.ravel_gated_mlp_grad_workspace(r(_mlp()), r(_mlp_grad(dx=None, dwg=None, dwu=None)), r(n)) == 0 and n.value == 0
    assert lib.ravel_gated_mlp_grad_workspace(r(_mlp()), r(_mlp_grad()), r(n)) == 0 and n.value >= 2 * 10 * 128 * 2
    for name, structs in (("ravel_norm_residual_grad", [_norm(), _norm_grad()]), ("ravel_cross_attention", [_cross()]),
                          ("ravel_cross_attention_grad", [_cross(), _cross_grad()]), ("ravel_gated_mlp", [_mlp()]),
                          ("ravel_gated_mlp_grad", [_mlp(), _mlp_grad()])):
        fn = getattr(lib, name + "_workspace")
        assert fn(*[r(s) for s in structs], None) == INVALID
        assert fn(*[None] * len(structs), r(n)) == INVALID


def test_nothing_wanted_is_nothing_done():
    """Gradients without outputs, and calls over no rows, come back without a launch (no GPU is needed to see it)."""
    none = dict(dx=None, df=None, dpost=None, dalpha=None, dgate=None, dscale=None, dshift=None)
    assert _call("ravel_norm_residual_grad", _norm(), _norm_grad(**none)) == 0
    assert _call("ravel_norm_residual", _norm(rows=0)) == 0
    assert _call("ravel_cross_attention_grad", _cross(), _cross_grad(dq=None, dk=None, dv=None)) == 0
    assert _call("ravel_cross_attention", _cross(rows=0)) == 0 and _call("ravel_cross_attention", _cross(batch=0)) == 0
    assert _call("ravel_gated_mlp", _mlp(rows=0)) == 0
    assert _call("ravel_gated_mlp_grad", _mlp(), _mlp_grad(dx=None, dwg=None, dwu=None)) == 0


def test_strides_of_single_rows_are_of_no_account():
    odd = 12345677
    assert _call("ravel_norm_residual_grad", _norm(rows=1, mods=1, x_out_stride=odd, f_stride=odd, gate_stride=odd, scale_stride=-7),
                 _norm_grad(dx=None, df=None, dpost=None, dalpha=None, dgate=None, dscale=None, dshift=None, dy_stride=odd)) == 0
    assert _call("ravel_cross_attention_grad", _cross(batch=1, rows=1, keys=1, q_stride=(odd, odd, 64), k_stride=(odd, odd, 64)),
                 _cross_grad(dq=None, dk=None, dv=None)) == 0


@pytest.mark.parametrize("struct,name", [("RavelNorm", "ravel_norm"), ("RavelNormGrad", "ravel_norm_grad"),
                                         ("RavelCross", "ravel_cross"), ("RavelCrossGrad", "ravel_cross_grad"),
                                         ("RavelMlp", "ravel_mlp"), ("RavelMlpGrad", "ravel_mlp_grad")])
def test_the_bindings_structures_are_the_headers(struct, name):
    ravel = _ravel()
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ravel.h")).read(), flags=re.S)
    body = re.search(r"typedef struct\s*\{([^}]*)\}\s*" + name + r"\s*;", text).group(1)
    want = []
    for kind, names in re.findall(r"(int32_t|int64_t|float|const int32_t\*|const void\*|void\*|const float\*|float\*)\s+([^;]+);", body):
        for n in names.split(","):
            m = re.match(r"\s*(\w+)(?:\[(\d+)\])?\s*$", n)
            c = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}.get(kind, ctypes.c_void_p)
            want.append((m.group(1), c * int(m.group(2)) if m.group(2) else c))
    assert getattr(ravel, struct)._fields_ == want
    pack = {"RavelNorm": ravel._pack_norm, "RavelNormGrad": ravel._pack_norm_grad, "RavelCross": ravel._pack_cross,
            "RavelCrossGrad": ravel._pack_cross_grad, "RavelMlp": ravel._pack_mlp, "RavelMlpGrad": ravel._pack_mlp_grad}[struct]
    n = sum(getattr(c, "_length_", 1) for _, c in want)
    assert len(pack(*range(n))) == ctypes.sizeof(getattr(ravel, struct))
    again = getattr(ravel, struct).from_buffer_copy(pack(*range(n)))
    flat = [x for f, c in want for x in (getattr(again, f) if hasattr(c, "_length_") else [getattr(again, f)])]
    assert [x or 0 for x in flat] == list(range(n))


def test_host_tensors_are_refused():
    import torch
    ravel = _ravel()
    x, w = torch.zeros((4, 64)), torch.zeros((8, 64))
    q = torch.zeros((1, 2, 2, 64))
    lse = torch.zeros((1, 2, 2))
    for call in (lambda: ravel.norm_residual(x), lambda: ravel.norm_residual_grad(x, x, x), lambda: ravel.cross_attention(q, q, q),
                 lambda: ravel.cross_attention_grad(q, q, q, q, lse, q), lambda: ravel.gated_mlp(x, w, w.clone()),
                 lambda: ravel.gated_mlp_grad(x, w, w.clone(), torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(4, 8))):
        with pytest.raises(ValueError, match="GPU"):
            call()
