"""Lanes past the rows of an activation hold no piece of it: every kernel has to look
at that before it reads codes and exponents (load_packed does not).  The optimiser may
sink such a read behind a later test and hide a mistake, so this reads what the
compiler makes of the source before any of its passes."""
import os
import re
import subprocess

import pytest

from paper_2609_06072_amd import build as b


def functions(text):
    """name -> [(label, instructions)] in order."""
    out = {}
    for m in re.finditer(r"^define [^@]*@([\w.$]+)\(.*?\{\n(.*?)^\}", text, re.M | re.S):
        blocks = [("entry", [])]
        for line in m.group(2).split("\n"):
            label = re.match(r"^([\w.]+):", line)
            if label:
                blocks.append((label.group(1), []))
            elif line.strip():
                blocks[-1][1].append(line.strip())
        out[m.group(1)] = blocks
    return out


def before_any_test(blocks):
    """The functions called before the first conditional branch."""
    at, calls, label, seen = dict(blocks), [], blocks[0][0], set()
    while label not in seen:
        seen.add(label)
        for line in at[label]:
            calls += re.findall(r"\bcall [^@]*@([\w.$]+)\(", line)
        last = at[label][-1]
        jump = re.match(r"br label %([\w.]+)", last)
        if not jump:
            break
        label = jump.group(1)
    return calls


def unguarded(text, reader="load_packed"):
    """Functions that call a reader before any test, themselves or through others."""
    early = {name: before_any_test(blocks) for name, blocks in functions(text).items()}
    found = {name for name in early if reader in name}
    assert found or reader not in text
    while True:
        more = {name for name, calls in early.items() if found & set(calls)} - found
        if not more:
            return found
        found |= more


def test_kernels_test_before_they_read_checkpoints(tmp_path):
    out = tmp_path / "k.ll"
    subprocess.run([b.hipcc(), *b.HIPFLAGS, "--cuda-device-only", "-S", "-emit-llvm", "-Xclang", "-disable-llvm-passes",
                    os.path.join(b.CSRC, "activation.hip"), "-o", str(out)], check=True, capture_output=True)
    text = out.read_text()
    # (not the functions made for one kernel, whose names hold its own)
    kernels = set(re.findall(r"^define amdgpu_kernel [^@]*@([\w.$]+)\(", text, re.M))
    assert len(kernels) == 2 * (1 + 1 + 3 + 2)
    assert any("load_packed" in n for n in functions(text))
    assert not kernels & unguarded(text)


PLANTED = """define void @load_packed_x(ptr %p) {
  %1 = load i8, ptr %p
  ret void
}
define void @through(ptr %p) {
  call void @load_packed_x(ptr %p)
  ret void
}
define void @kernel(ptr %p) {
BODY}
"""


@pytest.mark.parametrize("body,bad", [
    ("  call void @through(ptr %p)\n  ret void\n", True),
    ("  br label %a\n\na:\n  call void @through(ptr %p)\n  ret void\n", True),
    ("  br i1 %in, label %a, label %c\n\na:\n  call void @through(ptr %p)\n  br label %c\n\nc:\n  ret void\n", False),
    ("  ret void\n", False),
])
def test_scan_of_planted_reads(body, bad):
    assert ("kernel" in unguarded(PLANTED.replace("BODY", body))) == bad
