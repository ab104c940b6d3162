"""Matrix instructions written as assembly without wait states of their own
(mfma_ready): the compiler does not know that their operands must not come from
a vector instruction right before.  This reads the assembly of the library's own
source, backwards from each of them along every path."""
import os
import re
import subprocess

import pytest

from paper_2609_06072_amd import build as b
from test_matrix_waits import _functions, _parse

STATES = 2   # from a vector instruction's result to a matrix instruction's operand


def _regs(text, kind):
    regs = set()
    for lo, hi in re.findall(r"\b%s\[(\d+):(\d+)\]" % kind, text):
        regs |= set(range(int(lo), int(hi) + 1))
    return regs | {int(r) for r in re.findall(r"\b%s(\d+)\b" % kind, text)}


def unready(text):
    """Vector instructions that write an operand of an assembly-written matrix
    instruction within STATES before it."""
    ins, labels = _parse(text)
    at, jumps, found = {}, {}, []
    for label, i in labels.items():
        at.setdefault(i, []).append(label)
    for i, (op, line, _) in enumerate(ins):
        if "branch" in op:
            jumps.setdefault(line.split()[1], []).append(i)
    for i, (op, line, in_asm) in enumerate(ins):
        if not (in_asm and op.startswith("v_mfma")):
            continue
        operands = line.split(None, 1)[1]
        need_v, need_a = _regs(operands, "v"), _regs(operands, "a")
        work, seen = [(i, 0)], set()
        while work:
            j, t = work.pop()
            if t >= STATES or (j, t) in seen:
                continue
            seen.add((j, t))
            before = [j - 1] if j > 0 and ins[j - 1][0] != "s_branch" else []
            for label in at.get(j, []):
                before += jumps.get(label, [])
            for p in before:
                o, l, _ = ins[p]
                if o.startswith("v_") and not o.startswith("v_mfma"):
                    dst = l.split(None, 1)[1].split(",")[0]
                    if _regs(dst, "v") & need_v or _regs(dst, "a") & need_a:
                        found.append(f"{l}  ->  {line}")
                        continue
                work.append((p, t + (int(l.split()[1]) + 1 if o == "s_nop" else 1)))
    return found


def test_operands_are_ready(tmp_path):
    out = tmp_path / "k.s"
    subprocess.run([b.hipcc(), *b.HIPFLAGS, "--cuda-device-only", "-S", os.path.join(b.CSRC, "moe_gemm.hip"),
                    "-o", str(out)], check=True, capture_output=True)
    n = 0
    for name, text in _functions(out.read_text()):
        bad = unready(text)
        assert not bad, f"{name}: {len(bad)}, first {bad[0]}"
        n += "moe_dx_large" in name
    assert n == 2


MFMA = "\t;;#ASMSTART\n\tv_mfma_f32_16x16x32_bf16 a[8:11], v[0:3], v[4:7], a[8:11]\n\t;;#ASMEND\n"


@pytest.mark.parametrize("before,bad", [
    ("\tv_mov_b32_e32 v5, v9\n", True),
    ("\tv_mov_b32_e32 v9, v5\n", False),
    ("\tv_accvgpr_write_b32 a9, 0\n\ts_nop 0\n", True),
    ("\tv_accvgpr_write_b32 a9, 0\n\ts_nop 1\n", False),
    ("\tds_read_b128 v[4:7], v9\n", False),
    ("\tv_add_u32_e32 v4, v8, v9\n\ts_branch .L1\n\ts_nop 5\n.L1:\n", True),
    ("\tv_add_u32_e32 v4, v8, v9\n\ts_nop 5\n.L1:\n", False),
])
def test_scan_of_planted_hazards(before, bad):
    assert bool(unready(before + MFMA)) == bad
