"""The library's device code as it was built: wait states that the architecture asks for and that the compiler
cannot place in code written as asm; values moved for some lanes that all lanes read; addresses that only kernels have."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_17081_amd import build
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


def vectors(operand):
    """Names of the vector registers that an operand names."""
    m = re.match(r"([va])\[(\d+):(\d+)\]", operand) or re.match(r"([va])(\d+)\b", operand)
    return {m[1] + str(i) for i in range(int(m[2]), int(m[m.lastindex]) + 1)} if m else set()


def moved_for_some(instructions):
    """Moves of a vector register between the ends of two branches, one inside the other (so for lanes of the outer one alone), where the
    first instructions behind both write the register that was moved: what it held for the other lanes is lost."""
    out, last = [], None
    for i, (op, args) in enumerate(instructions):
        if op == "s_or_b64" and args[:2] == ["exec", "exec"]:
            for j in range(last + 1 if last is not None else i, i):
                name, given = instructions[j]
                if not (name.startswith(("v_mov_b", "v_accvgpr_")) and len(given) == 2 or name.startswith("scratch_store")):
                    continue
                moved = set().union(*(vectors(a) for a in (given[1:] if name.startswith("v_") else given)))
                for after, to in instructions[i + 1:i + 60]:
                    if "saveexec" in after or after.startswith(("s_cbranch", "s_branch", "s_endpgm")) or (after == "s_mov_b64" and to[0] == "exec"):
                        break
                    if after.startswith(("v_", "ds_read", "global_load", "buffer_load", "scratch_load")) and to and vectors(to[0]) & moved:
                        out.append(j)
                        break
            last = i
        elif op.startswith(("s_cbranch", "s_branch", "s_endpgm")) or "saveexec" in op or (args and args[0] == "exec"):
            last = None
    return out


# What was built of 17 rows of heads of 256 once: v[66:67], which all lanes read later, kept for the lanes of s[8:9] alone.
MOVED = """s_or_b64 exec, exec, s[10:11]
v_accvgpr_write_b32 a155, v67
v_accvgpr_write_b32 a154, v66
s_mov_b32 s94, s80
s_or_b64 exec, exec, s[8:9]
v_mov_b32_e32 v66, 0
v_mov_b32_e32 v67, v66
s_and_saveexec_b64 s[8:9], s[0:1]"""


@pytest.mark.parametrize("text,want", [
    (MOVED, [1, 2]), (MOVED.replace("v66, 0", "v68, 0"), [1]), (MOVED.replace("s[8:9]\nv_mov", "s[8:9]\ns_cbranch_execz 5\nv_mov"), []),
    (MOVED.replace("s_mov_b32 s94, s80", "s_and_saveexec_b64 s[10:11], vcc"), []),
    ("s_or_b64 exec, exec, s[2:3]\nscratch_store_dwordx2 off, v[4:5], off\ns_or_b64 exec, exec, s[0:1]\nds_read_b32 v5, v1", [1]),
    ("s_or_b64 exec, exec, s[10:11]\nv_accvgpr_read_b32 v34, a176\ns_or_b64 exec, exec, s[8:9]\nv_mov_b32_e32 v34, 0", [])])
def test_moved_for_some_by_hand(text, want):
    assert moved_for_some(parse(text)) == want


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


def test_no_values_moved_for_some_lanes(tmp_path):
    """In attention, whose kernels move many registers.  (Elsewhere such moves are the source's own: y = x for some, then x = z.)"""
    tool = objdump()
    if not tool or not rk.library_available():
        pytest.skip("no llvm-objdump, or the library is not built")
    so = shutil.copy(rk.LIB_PATH, tmp_path)
    subprocess.run([tool, "--offloading", so], cwd=tmp_path, check=True, capture_output=True)
    ends, wrong = 0, []
    for f in sorted(glob.glob(os.path.join(str(tmp_path), "*gfx950"))):
        text = subprocess.run([tool, "-d", "--no-show-raw-insn", f], check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\w*attend_kernel\w*)>:\n(.*?)(?=^[0-9a-f]+ <|\Z)", text, re.M | re.S):
            code = parse(body)
            ends += sum(op == "s_or_b64" and args[:2] == ["exec", "exec"] for op, args in code)
            wrong += [(name, *code[j]) for j in moved_for_some(code)]
    assert ends > 0 and not wrong, (ends, len(wrong), wrong[:5])


def test_only_kernels_ask_for_their_arguments_address(tmp_path):
    """Where a function that a kernel calls asks for the address of the kernel's arguments, it gets 0.  Without optimization all is
    called that need not be inlined."""
    try:
        cc = build.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    flags = [f for f in build.HIPCC_FLAGS if f != "-O3"]
    asked, outside = 0, []
    for src in build.SOURCES:
        text = open(os.path.join(build.CSRC, src)).read()
        if "kernarg_segment_ptr" not in text:
            continue
        to = str(tmp_path / "out.ll")
        subprocess.run([cc, *flags, "-O0", "--offload-device-only", "-emit-llvm", "-S", os.path.join(build.CSRC, src), "-o", to],
                       check=True, capture_output=True)
        for line in open(to):
            if line.startswith("define"):
                where = line
            elif "llvm.amdgcn.kernarg.segment.ptr" in line and " call " in line:
                asked += 1
                outside += [] if "amdgpu_kernel" in where else [re.search(r"@(\w+)", where)[1]]
    assert asked > 0 and not outside, (asked, sorted(set(outside))[:5])
