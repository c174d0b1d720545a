"""Wait states that the processor does not see to by itself, counted in the machine code of the built library.  The compiler puts
them between its own instructions but does not look into inline assembly."""
import os
import re
import shutil
import subprocess

import pytest

from paper_1611_06256_amd import binding

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def _registers(operands):
    got = {int(r) for r in re.findall(r"\bs(\d+)\b", operands)}
    for a, b in re.findall(r"\bs\[(\d+):(\d+)\]", operands):
        got |= set(range(int(a), int(b) + 1))
    return got | ({106, 107} if "vcc" in operands else set())


def _needs(before, ins):
    """What is missing in front of a vector memory instruction, given the instructions before it, the last one at the end."""
    if " lds" in ins or "_lds_" in ins:
        # a scalar write of m0, and a load to LDS, whose place m0 gives: one state between them
        if before and re.match(r"s_\w+ m0,", before[-1]):
            return "m0"
    reads, states = _registers(ins), 0
    for b in reversed(before):
        if states >= 5:                 # a vector instruction that writes a scalar register, and its reader: five
            return None
        op, _, rest = b.partition(" ")
        if op.startswith("v_") and reads & _registers(rest.split(",")[0]):
            return "scalar register of a vector instruction"
        states += 1 + int(rest) if op == "s_nop" else 1
    return None


def test_the_rule_itself():
    load = "global_load_lds_dwordx4 v1, s[2:3]"
    assert _needs(["s_mov_b32 m0, s9"], load) == "m0"
    assert _needs(["s_mov_b32 m0, s9", "s_nop 0"], load) is None
    assert _needs(["v_readfirstlane_b32 s3, v0", "s_nop 0"], load)
    assert _needs(["v_readfirstlane_b32 s3, v0", "s_nop 3"], load)
    assert _needs(["v_readfirstlane_b32 s3, v0", "s_nop 4"], load) is None
    assert _needs(["v_readfirstlane_b32 s4, v0"], load) is None
    assert _needs(["s_mov_b32 m0, s9"], "global_load_dwordx4 v[0:3], v1, s[2:3]") is None


def test_memory_instructions_have_their_wait_states(tmp_path):
    binding.load_library()
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    shutil.copy(binding.lib_path(), tmp_path / "lib.so")
    subprocess.check_call([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, stdout=subprocess.DEVNULL)
    objects = [f for f in os.listdir(tmp_path) if f.endswith("gfx950")]
    assert objects
    missing, to_lds = {}, 0
    for f in objects:
        text = subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", f], cwd=tmp_path, stdout=subprocess.PIPE, text=True).stdout
        kernel, before = None, []
        for line in text:
            if line.rstrip().endswith(">:"):
                kernel, before = line.split("<")[1].split(">")[0], []
                continue
            ins = line.split("//")[0].strip()
            if not ins:
                continue
            if ins.startswith(("global_", "buffer_", "flat_", "scratch_")):
                to_lds += " lds" in ins or "_lds_" in ins
                what = _needs(before, ins)
                if what:
                    missing.setdefault((kernel, what), (before[-6:], ins))
            before.append(ins)
            del before[:-8]
    assert to_lds > 100
    assert not missing, f"{len(missing)} kernels, for instance {next(iter(missing.items()))}"
