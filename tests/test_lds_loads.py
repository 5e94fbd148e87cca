"""Loads from memory straight into LDS take their LDS address from M0, and need
one wait state after a scalar write of it.  The compiler's hazard pass does not
look into asm strings, so the built library is read back: nowhere is such a load
the instruction right behind a write of M0.  CPU only."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_17652_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
LOAD = re.compile(r"(global|buffer|scratch)_load_lds_|buffer_load_\w+ .* lds\b")
WRITES_M0 = re.compile(r"s_\w+ m0\b")


def faults(lines):
    """(how many loads to LDS, the first lines of those without a wait state)"""
    loads, bad, last = 0, [], ""
    for line in lines:
        text = line.split("//")[0].strip()
        if not text or text.endswith(":"):
            continue
        if LOAD.match(text):
            loads += 1
            if WRITES_M0.match(last):
                bad.append((last, text))
        last = text
    return loads, bad


def test_the_reader_itself():
    ok = ["\ts_mov_b32 m0, s4 // 0", "\ts_nop 0", "\tglobal_load_lds_dwordx4 v1, s[2:3]"]
    assert faults(ok) == (1, [])
    assert len(faults([ok[0], ok[2]])[1]) == 1
    assert len(faults(["s_add_i32 m0, s0, 0", "buffer_load_dword v1, s[0:3], 0 offen lds"])[1]) == 1


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler here")
def test_a_wait_state_lies_between_m0_and_every_load_to_lds(tmp_path):
    if not os.path.exists(build.LIB_PATH):
        build.build()
    lib = shutil.copy(build.LIB_PATH, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, stdout=subprocess.DEVNULL)
    total = 0
    for code in sorted(glob.glob(os.path.join(tmp_path, "*" + build.ARCH))):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", code], check=True,
                              capture_output=True, text=True).stdout
        loads, bad = faults(text.splitlines())
        assert not bad, (os.path.basename(code), len(bad), bad[:3])
        total += loads
    assert total > 1000          # attention, the LM head and the 4-bit linear layers
