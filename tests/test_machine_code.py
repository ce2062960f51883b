"""The built library leaves the wait states that matrix instructions need, along every path (tests/machine_code.py)."""

import os
import shutil

import pytest

from tests import machine_code as mc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_34170_amd", "libravel.so")


def _code(lines):
    """A listing as the disassembler prints it, 4 bytes an instruction; a branch's operand is the instructions that it skips."""
    return mc.kernel([f"\t{text} // {4 * i:012X}: 00000000" for i, text in enumerate(lines)])


PRODUCT = "v_mfma_f32_16x16x32_bf16 v[0:3], v[8:11], v[12:15], v[0:3]"


@pytest.mark.parametrize("between,use,states", [
    (["s_nop 6"], "v_add_f32_e32 v20, v21, v3", 7),
    (["s_nop 6"], "v_mov_b32_e32 v2, 0", 7),
    (["s_nop 2", "v_mov_b32_e32 v30, 0"], "global_store_dwordx4 v[40:41], v[0:3], off", 4),
    (["s_cbranch_scc1 2", "s_nop 7", "s_nop 7"], "v_mul_f32_e32 v20, 2.0, v0", 1),  # the wait is skipped
    (["s_nop 3", "s_branch 1", "s_nop 7"], "v_mfma_f32_16x16x32_bf16 v[4:7], v[0:3], v[12:15], v[4:7]", 5),
    ([], "v_permlane32_swap_b32_e32 v20, v1", 0),
    ([], "ds_write_b128 v30, v[0:3]", 0),
    ([], "v_accvgpr_write_b32 a0, v3", 0),
])
def test_uses_that_are_too_early(between, use, states):
    found = mc.too_early(_code([PRODUCT, *between, use, "s_endpgm"]))
    assert [(f[1], f[2], f[3]) for f in found] == [(use, states, 8)]


@pytest.mark.parametrize("lines", [
    [PRODUCT, "s_nop 7", "v_add_f32_e32 v20, v21, v3"],
    [PRODUCT, "s_cbranch_scc1 1", "s_nop 7", "s_nop 6", "v_mul_f32_e32 v20, 2.0, v0"],
    [PRODUCT, "v_mfma_f32_16x16x32_bf16 v[0:3], v[16:19], v[12:15], v[0:3]", "s_nop 7", "v_mov_b32_e32 v20, v0"],  # a sum that goes on
    [PRODUCT, "v_mov_b32_e32 v8, v20", "s_add_u32 s0, s1, s2", "v_mov_b32_e32 v21, a0"],  # other registers
    [PRODUCT, "s_branch 2", "v_mov_b32_e32 v20, v0", "s_endpgm", "s_nop 7", "v_mov_b32_e32 v20, v0"],
])
def test_uses_that_are_not(lines):
    assert mc.too_early(_code(lines + ["s_endpgm"])) == []


def test_loops_are_followed_around():
    code = _code(["v_mov_b32_e32 v20, v0", "s_nop 3", PRODUCT, "s_cbranch_scc1 65532", "s_endpgm"])
    assert [(f[1], f[2]) for f in mc.too_early(code)] == [("v_mov_b32_e32 v20, v0", 1)]


@pytest.mark.skipif(not os.path.exists(LIB), reason="libravel.so not built")
@pytest.mark.skipif(not os.path.exists(os.path.join(mc.TOOLS, "llvm-objdump")), reason="no disassembler")
def test_the_library(tmp_path):
    names, bad = set(), []
    for name, lines in mc.functions(LIB, str(tmp_path)):
        names.add(name)
        bad += [(name, *f) for f in mc.too_early(mc.kernel(lines))]
    shutil.rmtree(tmp_path)
    for part in ("cross_kernel", "cross_dq_kernel", "cross_dkv_kernel", "cross_few_keys_grad_kernel", "mlp_matrix_kernel", "mlp_rows_kernel"):
        assert any(part in n for n in names), part
    assert not bad, (len(bad), bad[:4])
