"""CPU check of a gfx950 hazard that the compiler does not see inside assembly
text: a scalar register written by a vector instruction (v_readlane of a
spilled address, v_readfirstlane) must be five wait states ahead of a
vector-memory instruction that reads it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_15160_amd import build, tlf

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
INSTRUCTION = re.compile(r"\s+([a-z]\w+)\s*([^/]*)")


def scalars(text):
    """Numbers of the scalar registers named in an operand list."""
    found = {int(n) for n in re.findall(r"\bs(\d+)\b", text)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        found |= set(range(int(a), int(b) + 1))
    return found


def too_close(lines):
    """(writer, reader) pairs of a straight run of instructions with fewer than five wait states between them."""
    recent, bad = [], []
    for line in lines:
        m = INSTRUCTION.match(line)
        if not m:
            recent = []
            continue
        op, args = m[1], m[2].strip()
        if re.match(r"(global|buffer|scratch|flat)_", op):
            waits = 0
            for o, a in reversed(recent):
                if waits >= 5:
                    break
                if re.match(r"v_read(first)?lane", o) and scalars(a.split(",")[0]) & scalars(args):
                    bad.append((f"{o} {a}", f"{op} {args}"))
                waits += int(a, 0) + 1 if o == "s_nop" else 1
        recent = (recent + [(op, args)])[-8:]
    return bad


def test_the_check_finds_a_planted_pair():
    near = ["\tv_readlane_b32 s17, v250, 25", "\ts_nop 0", "\tglobal_load_lds_dwordx4 v2, s[16:17]"]
    far = ["\tv_readlane_b32 s17, v250, 25", "\ts_nop 4", "\tglobal_load_lds_dwordx4 v2, s[16:17]"]
    assert len(too_close(near)) == 1 and not too_close(far)


def test_scalar_addresses_are_waited_for(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    if not os.path.exists(tlf.LIB_PATH):
        build.build()
    lib = shutil.copy(tlf.LIB_PATH, tmp_path)
    subprocess.check_call([OBJDUMP, "--offloading", lib], cwd=tmp_path, stdout=subprocess.DEVNULL)
    bad = []
    for name in sorted(os.listdir(tmp_path)):
        if name.endswith("gfx950"):
            text = subprocess.check_output([OBJDUMP, "-d", "--no-show-raw-insn", str(tmp_path / name)], text=True)
            bad += too_close(text.splitlines())
    assert not bad, bad[:5]
