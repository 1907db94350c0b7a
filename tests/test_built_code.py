"""The library's device code as it was built: wait states that the architecture asks for and that the compiler
cannot place in code written as asm."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_17081_amd import rkroute as rk

WAIT_M0 = 1            # between a scalar write of m0 and a load to LDS, which reads it
WAIT_SGPR = 5          # between a vector instruction's write of a scalar register and a vector memory instruction that reads it


def objdump():
    found = shutil.which("llvm-objdump")
    for root in (os.environ.get("ROCM_PATH", "/opt/rocm"), "/opt/rocm"):
        found = found or shutil.which(os.path.join(root, "llvm", "bin", "llvm-objdump"))
    return found


def scalars(operand):
    """Numbers of the scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand) or re.fullmatch(r"s(\d+)", operand)
    return set(range(int(m[1]), int(m[m.lastindex]) + 1)) if m else set()


def writes_m0(op, args):
    return op.startswith("s_") and not op.startswith("s_cmp") and args[:1] == ["m0"]


def faults(instructions):
    """Loads to LDS of a straight list of (name, operands) that follow too closely on what they read."""
    out = []
    for i, (op, args) in enumerate(instructions):
        if not (op.startswith("buffer_load") and args and args[-1].split()[-1] == "lds"):
            continue
        reads = set().union(*(scalars(a.split()[0]) for a in args if a))
        waits, j = 0, i - 1
        while j >= 0 and waits < WAIT_SGPR:
            name, given = instructions[j]
            if name == "s_nop":
                waits += int(given[0], 0) + 1
            else:
                if waits < WAIT_M0 and writes_m0(name, given):
                    out.append((i, "m0"))
                if name.startswith("v_") and given and scalars(given[0]) & reads:
                    out.append((i, "descriptor"))
                waits += 1
            j -= 1
    return out


def parse(text):
    got = []
    for line in text.splitlines():
        line = line.split("//")[0].strip()
        m = re.match(r"([a-z_][a-z_0-9]+)(?:\s+(.*))?$", line)
        if m:
            got.append((m[1], [a.strip() for a in m[2].split(",")] if m[2] else []))
    return got


@pytest.mark.parametrize("text,want", [
    ("s_mov_b32 m0, s3\nbuffer_load_dwordx4 v1, s[4:7], 0 offen lds", ["m0"]),
    ("s_mov_b32 m0, s3\ns_nop 0\nbuffer_load_dwordx4 v1, s[4:7], 0 offen lds", []),
    ("v_readlane_b32 s6, v1, 2\ns_mov_b32 m0, s3\ns_nop 2\nbuffer_load_dwordx4 v1, s[4:7], 0 offen lds", ["descriptor"]),
    ("v_readlane_b32 s6, v1, 2\ns_mov_b32 m0, s3\ns_nop 3\nbuffer_load_dwordx4 v1, s[4:7], 0 offen lds", []),
    ("s_mov_b32 m0, s3\nbuffer_load_dwordx4 v[0:3], v4, s[4:7], 0 offen", []),
])
def test_faults_by_hand(text, want):
    assert [w for _, w in faults(parse(text))] == want


def test_loads_to_lds_wait_for_what_they_read(tmp_path):
    tool = objdump()
    if not tool or not rk.library_available():
        pytest.skip("no llvm-objdump, or the library is not built")
    so = shutil.copy(rk.LIB_PATH, tmp_path)
    subprocess.run([tool, "--offloading", so], cwd=tmp_path, check=True, capture_output=True)
    loads, wrong = 0, []
    for f in sorted(glob.glob(os.path.join(str(tmp_path), "*gfx950"))):
        text = subprocess.run([tool, "-d", "--no-show-raw-insn", f], check=True, capture_output=True, text=True).stdout
        code = parse(text)
        loads += sum(op.startswith("buffer_load") and args[-1].split()[-1] == "lds" for op, args in code if args)
        wrong += faults(code)
    assert loads > 0 and not wrong, (loads, len(wrong), wrong[:5])
