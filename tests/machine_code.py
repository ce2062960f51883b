"""Distances between matrix instructions and the use of their results, in the gfx950 code of a library built here.

The hardware does not hold back a vector instruction that reads or overwrites a matrix instruction's result too early: the
program has to leave wait states between them (every instruction is one, s_nop N is N + 1).  The compiler counts them, but not
along every path: wrong sums have been seen where a uniform branch skipped a few instructions.  Here every path is walked.
"""

import os
import re
import subprocess

TOOLS = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")

# Wait states from a result to its first use outside matrix instructions' sums: 16 x 16 x 32 bf16 products take 4 passes of 4
# clocks, 32 x 32 x 16 ones 8, the 32-bit ones 8 on the slower pipe.
STATES = {"v_mfma_f32_16x16x16_bf16": 8, "v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_32x32x16_bf16": 12,
          "v_mfma_f32_16x16x4_f32": 10}
FURTHEST = max(STATES.values())
_VECTOR = ("v_", "ds_", "buffer_", "global_", "flat_", "scratch_")
_REG = re.compile(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+)\b)")


def _registers(text):
    r = set()
    for kind, lo, hi, one in _REG.findall(text):
        r.update((kind, i) for i in (range(int(lo), int(hi) + 1) if lo else (int(one),)))
    return frozenset(r)


class Instruction:
    __slots__ = ("op", "reads", "writes", "states", "next", "text")

    def __init__(self, text):
        self.text = text
        self.op, _, args = text.partition(" ")
        self.reads = self.writes = frozenset()
        self.states = int(args) + 1 if self.op == "s_nop" else 1
        if not self.op.startswith(_VECTOR):
            return
        args = args.split(", ")
        if "mfma" in self.op:  # (the sums' operand, the last one, is forwarded)
            self.writes, self.reads = _registers(args[0]), _registers(" ".join(args[1:3]))
        elif "store" in self.op or self.op.startswith("ds_write") or args[-1].endswith(" lds"):
            self.reads = _registers(" ".join(args))
        else:
            both = self.op.startswith(("v_swap", "v_permlane16_swap", "v_permlane32_swap", "v_fmac", "v_pk_fmac", "v_dot"))
            dpp = "row_" in text or "quad_perm" in text  # (lanes that are masked keep the old value)
            self.writes = _registers(args[0])
            self.reads = _registers(" ".join(args if both or dpp else args[1:]))


def kernel(lines):
    """Instructions of a disassembled function, each with those that may follow it."""
    code, at, jumps = [], {}, []
    for line in lines:
        text, _, note = line.partition("//")
        address = re.match(r"\s*([0-9A-F]+):", note)
        at[int(address.group(1), 16)] = len(code)
        i = Instruction(" ".join(text.split()))
        if i.op == "s_branch" or i.op.startswith("s_cbranch"):
            jumps.append((len(code), int(address.group(1), 16) + 4 + 4 * _signed(int(i.text.split()[1]))))
        code.append(i)
    for n, i in enumerate(code):
        i.next = [n + 1] if n + 1 < len(code) and i.op not in ("s_branch", "s_endpgm") else []
    for n, target in jumps:
        code[n].next.append(at[target])
    return code


def _signed(n):
    return n - 65536 if n >= 32768 else n


def too_early(code):
    """(matrix instruction, first use, states between them, states needed) of every result that is used too early."""
    found = []
    for i in code:
        if "mfma" not in i.op:
            continue
        need = STATES[i.op]
        seen, paths = {}, [(n, 0, i.writes) for n in i.next]
        while paths:
            n, states, live = paths.pop()
            if states >= need or not live or seen.get((n, live), FURTHEST) <= states:
                continue
            seen[n, live] = states
            j = code[n]
            if "mfma" in j.op:
                if j.reads & live:
                    found.append((i.text, j.text, states, need))
                    continue
                live -= j.writes  # (sums that go on have been waited for by the hardware)
            elif (j.reads | j.writes) & live:
                found.append((i.text, j.text, states, need))
                continue
            paths += [(m, states + j.states, live) for m in j.next]
    return found


def functions(library, folder):
    """(name, disassembled lines) of the functions of a library's gfx950 code that hold matrix instructions; `folder` takes
    the code objects."""
    link = os.path.join(folder, "library.so")
    os.symlink(os.path.abspath(library), link)
    subprocess.run([os.path.join(TOOLS, "llvm-objdump"), "--offloading", link], cwd=folder, check=True, capture_output=True)
    for name in sorted(os.listdir(folder)):
        if not name.endswith("gfx950"):
            continue
        text = subprocess.run([os.path.join(TOOLS, "llvm-objdump"), "-d", "--no-show-raw-insn", name], cwd=folder, check=True,
                              capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]{16} <)", text):
            head, _, body = part.partition("\n")
            m = re.match(r"[0-9a-f]{16} <(\w+)>:", head)
            if m and "v_mfma" in body:
                yield m.group(1), [line for line in body.split("\n") if "//" in line]
