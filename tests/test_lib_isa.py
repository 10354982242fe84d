"""The built library's gfx950 code: hazards that the compiler does not see inside inline assembly."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2510_18830_amd import build as B

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    """Lists of instructions, one for each code object of the library."""
    if OBJDUMP is None or not os.path.exists(B.LIB_PATH):
        pytest.skip("no llvm-objdump, or the library is not built")
    at = tmp_path_factory.mktemp("isa")
    lib = str(at / "libmsparse.so")
    shutil.copyfile(B.LIB_PATH, lib)
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=at, check=True, capture_output=True)
    objects = sorted(p for p in os.listdir(at) if p.endswith(B.ARCH))
    assert objects
    out = []
    for p in objects:
        text = subprocess.run([OBJDUMP, "-d", f"--mcpu={B.ARCH}", str(at / p)], check=True, capture_output=True, text=True)
        out.append([re.sub(r"\s*//.*", "", x).strip() for x in text.stdout.splitlines() if "//" in x])
    return out


def _hazards(instructions):
    """Loads into LDS that directly follow a scalar write of M0, which they read: one wait state has to lie between."""
    writes = re.compile(r"s_\w+ m0\b")
    reads = re.compile(r"(global|buffer|scratch)_load_\S*lds|(global|buffer|scratch)_load.*\blds\b|ds_\w*addtid|s_sendmsg")
    return [f"{a}; {b}" for a, b in zip(instructions, instructions[1:]) if writes.match(a) and reads.match(b)]


def test_hazards_are_found():
    load = "global_load_lds_dwordx4 v[0:1], off"
    assert _hazards(["s_mov_b32 m0, s4", load]) and _hazards(["s_add_u32 m0, s4, 16", "buffer_load_dword v1, s[0:3], 0 lds"])
    assert not _hazards(["s_mov_b32 m0, s4", "s_nop 0", load]) and not _hazards(["s_mov_b32 s0, m0", load])


def test_loads_into_lds_wait_for_m0(code):
    loads = sum("load_lds" in x for instructions in code for x in instructions)
    assert loads > 100
    found = [x for instructions in code for x in _hazards(instructions)]
    assert not found, f"{len(found)} of {loads}: {found[:3]}"


def _scalars(operand):
    """The scalar registers of an operand, as numbers (vcc: -1)."""
    m = re.fullmatch(r"s(\d+)|s\[(\d+):(\d+)\]|(vcc)\S*", operand)
    if not m:
        return set()
    if m.group(4):
        return {-1}
    return {int(m.group(1))} if m.group(1) else set(range(int(m.group(2)), int(m.group(3)) + 1))


def _late_scalars(instructions):
    """Memory instructions within five wait states of a vector instruction's write of a scalar register that they read."""
    found, recent = [], []   # (registers written, wait states since)
    for x in instructions:
        name, _, rest = x.partition(" ")
        operands = [o.strip() for o in rest.replace(" ", ",").split(",") if o]
        if re.match(r"global_|buffer_|flat_|scratch_", name):
            reads = set().union(*(_scalars(o) for o in operands)) if operands else set()
            found += [f"{x}: written {n} before" for regs, n in recent if regs & reads]
        states = int(operands[0], 0) + 1 if name == "s_nop" else 1
        recent = [(regs, n + states) for regs, n in recent if n + states < 5]
        if name.startswith("v_") and operands:
            written = _scalars(operands[0]) | (_scalars(operands[1]) if "_co_" in name and len(operands) > 1 else set())
            if written:
                recent.append((written, 0))
    return found


def test_late_scalars_are_found():
    write, load = "v_readlane_b32 s5, v1, s0", "global_load_lds_dwordx4 v0, s[4:5]"
    assert _late_scalars([write, "s_nop 3", load]) and _late_scalars([write, "s_mov_b32 m0, s1", "s_nop 0", load])
    assert not _late_scalars([write, "s_nop 4", load]) and not _late_scalars([write, "global_load_dword v0, v1, s[6:7]"])


def test_memory_instructions_wait_for_scalars(code):
    found = [x for instructions in code for x in _late_scalars(instructions)]
    assert not found, found[:5]
