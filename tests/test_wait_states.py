"""Wait states that the hardware asks for and that no pass of the compiler puts into inline assembly, in the library's own code as it was built.

A load into LDS takes its place from M0: between a scalar write of M0 and the load stands one instruction at least (gfx9 family: "SALU writes M0", then an LDS-DMA
load, one wait state).  A vector instruction's write of a scalar register stands five wait states before a memory instruction that reads it."""
import os
import re
import subprocess

import pytest

from paper_2406_09904_amd import binding

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
DMA = re.compile(r"global_load_lds_\w+|buffer_load_\w+.*\blds\b")


def _registers(text):
    """Scalar registers that are named: s5, s[4:7], vcc."""
    found = {int(n) for n in re.findall(r"\bs(\d+)\b", text)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", text):
        found |= set(range(int(a), int(b) + 1))
    return found | ({"vcc"} if "vcc" in text else set())


def _wait_states(line):
    return 1 + int(line.split()[1]) if line.startswith("s_nop") else 1


def faults(lines):
    """(what, the two instructions) of a disassembly's lines, one instruction each."""
    found = []
    for i, line in enumerate(lines):
        if not DMA.match(line):
            continue
        if re.match(r"s_\w+ m0\b", lines[i - 1]):
            found.append(("M0", lines[i - 1], line))
        reads, states = _registers(line), 0
        for before in reversed(lines[max(i - 5, 0):i]):
            if states >= 5 or before.endswith(":"):
                break
            to = before.split(" ", 1)[1].split(",")[0] if " " in before else ""
            if before.startswith("v_") and re.match(r"s\d|s\[|vcc", to) and _registers(to) & reads:
                found.append(("scalar", before, line))
            states += _wait_states(before)
    return found


def test_what_counts_as_a_fault():
    load = "global_load_lds_dwordx4 v3, s[4:5]"
    assert faults(["s_mov_b32 m0, s3", load]) and faults(["s_add_i32 m0, s3, 4", load])
    assert not faults(["s_mov_b32 m0, s3", "s_nop 0", load]) and not faults(["s_mov_b32 m0, s3", "v_add_u32 v3, v3, v4", load])
    assert faults(["v_readlane_b32 s5, v9, 3", "s_mov_b32 m0, s3", "s_nop 0", load]) and not faults(["v_readlane_b32 s5, v9, 3", "s_mov_b32 m0, s3", "s_nop 3", load])
    assert not faults(["v_readlane_b32 s6, v9, 3", "s_mov_b32 m0, s3", "s_nop 0", load])


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump beside the compiler")
def test_loads_into_lds_come_late_enough(tmp_path):
    if not os.path.exists(binding.LIB_PATH):
        from paper_2406_09904_amd import build
        build.build()
    os.symlink(binding.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    loads = 0
    for name in sorted(os.listdir(tmp_path)):
        if not name.endswith("gfx950"):
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", name], cwd=tmp_path, check=True, capture_output=True, text=True).stdout
        lines = [" ".join(l.split("//")[0].split()) for l in text.splitlines()]
        lines = [l for l in lines if l]
        loads += sum(bool(DMA.match(l)) for l in lines)
        found = faults(lines)
        assert not found, (name, len(found), found[:3])
    assert loads > 1000
