"""Wait states around loads that go straight into LDS, in the machine code of
the built library.

These loads are written as inline assembly, where the compiler adds no wait
states.  The target wants one instruction (or s_nop) between a scalar write of
m0 and a load into LDS, which takes its LDS address from m0, and five wait
states between a vector instruction that writes a scalar register and a memory
instruction that reads it (a buffer's descriptor)."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2608_08330_amd import build as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def scalars(operand):
    """Numbers of the scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return range(int(m[1]), int(m[2]) + 1)
    m = re.fullmatch(r"s(\d+)", operand)
    return (int(m[1]),) if m else ()


def hazards(lines):
    """(kind, function, instruction) of every missing wait, and the number of
    loads into LDS."""
    found, loads, function, before, age = [], 0, "", "", {}
    for line in lines:
        if not line.startswith("\t"):
            m = re.match(r"[0-9a-f]+ <(.*)>:", line)
            if m:
                function, before, age = m[1], "", {}
            continue
        text = line.split("//")[0].strip()
        op, _, rest = text.partition(" ")
        operands = rest.replace(",", " ").split()
        if op.startswith(("buffer_", "global_")):
            if "lds" in operands or "_lds_" in op:
                loads += 1
                if re.match(r"s_\w+ m0\b", before):
                    found.append(("m0", function, text))
            found += [("scalar", function, text) for x in operands for r in scalars(x) if r in age]
        waits = int(operands[0], 0) + 1 if op == "s_nop" else 1
        age = {r: n + waits for r, n in age.items() if n + waits < 5}
        if op.startswith(("v_readfirstlane", "v_readlane", "v_cmp")):
            age.update((r, 0) for r in scalars(operands[0]))
        before = text
    return found, loads


def test_the_scan_sees_both_hazards():
    load = "\tbuffer_load_dwordx4 v1, s[4:7], 0 offen lds // 0"
    head = ["0000 <f>:"]
    assert hazards(head + ["\ts_mov_b32 m0, s3", load])[0][0][0] == "m0"
    assert hazards(head + ["\ts_add_u32 m0, s3, 0x400", "\tglobal_load_lds_dwordx4 v[0:1], off"])[0][0][0] == "m0"
    assert hazards(head + ["\ts_mov_b32 m0, s3", "\ts_nop 0", load]) == ([], 1)
    assert hazards(head + ["\tv_readfirstlane_b32 s5, v0", "\ts_nop 3", load])[0][0][0] == "scalar"
    assert hazards(head + ["\tv_readfirstlane_b32 s5, v0", "\ts_nop 4", load]) == ([], 1)


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_loads_into_lds_wait_for_their_scalars(tmp_path):
    library = os.path.join(B.LIB, "librtcc.so")
    if not os.path.exists(library):
        B.build()
    shutil.copy(library, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    loads = 0
    for name in sorted(os.listdir(tmp_path)):
        if B.ARCH in name and os.path.getsize(tmp_path / name):
            text = subprocess.run([OBJDUMP, "-d", name], cwd=tmp_path, check=True, stdout=subprocess.PIPE, text=True).stdout
            found, n = hazards(text.splitlines())
            assert not found, (len(found), found[0])
            loads += n
    assert loads > 0
