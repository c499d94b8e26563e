"""Waits that the compiler does not count: direct global -> LDS loads are issued from inline assembly, inside of which it
inserts none for the registers that the instructions before have written.  The built kernels' own code is read; no GPU is
needed.

  M0 (the LDS address) written by a scalar or vector instruction: one wait state before the load;
  an address in scalar registers written by a vector instruction: five.
An instruction is one wait state, s_nop n is n + 1."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2608_06849_amd import aoh as A

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin" + os.pathsep + os.environ.get("PATH", ""))


def registers(operand):
    """Names of the scalar registers of an operand."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return {f"s{i}" for i in range(int(m[1]), int(m[2]) + 1)}
    return {operand} if re.fullmatch(r"s\d+|m0", operand) else set()


def split(line):
    """Mnemonic and operands of a line of the listing."""
    words = line.split(None, 1)
    return words[0], [w.strip() for w in words[1].split(",")] if len(words) > 1 else []


def short_waits(code):
    """Loads of a listing (instructions, labels as None) that come too early, and the number of loads."""
    found, loads = [], 0
    for i, line in enumerate(code):
        if line is None or not (line.startswith("global_load_lds") or (line.startswith("buffer_load") and line.endswith(" lds"))):
            continue
        loads += 1
        address = set().union(*(registers(x.split()[0]) for x in split(line)[1] if x))
        states, at = 0, i - 1
        while at >= 0 and states < 5:
            if code[at] is not None:
                op, operands = split(code[at])
                written = registers(operands[0]) if operands else set()
                if ("m0" in written and states < 1) or (op.startswith("v_") and written & address):
                    found.append(f"{code[at]} / {line}")
                    break
                states += int(operands[0], 0) + 1 if op == "s_nop" else 1
            at -= 1
    return found, loads


def test_the_reading_itself():
    load = "global_load_lds_dwordx4 v1, s[4:5]"
    for code, bad in ((["s_mov_b32 m0, s1", load], 1), (["v_readfirstlane_b32 m0, v2", load], 1), (["s_mov_b32 m0, s1", "s_nop 0", load], 0),
                      (["s_mov_b32 m0, s1", "v_add_u32_e32 v3, v4, v5", load], 0), (["s_mov_b32 s4, s1", load], 0),
                      (["v_readfirstlane_b32 s5, v2", "s_mov_b32 m0, s1", "s_nop 0", load], 1),
                      (["v_readfirstlane_b32 s5, v2", "s_mov_b32 m0, s1", None, "s_nop 3", load], 0),
                      (["v_readlane_b32 s4, v2, 3", "s_nop 4", load], 0), (["v_readlane_b32 s4, v2, 3", "s_nop 3", load], 1),
                      (["v_readlane_b32 s6, v2, 3", load], 0), (["s_add_i32 m0, s2, s3", "buffer_load_dwordx4 v1, s[8:11], 0 offen lds"], 1)):
        assert short_waits(code) == ([f"{code[0]} / {code[-1]}"] * bad, 1), code


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_direct_loads_wait_for_their_addresses(tmp_path):
    library = shutil.copy(A.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", library], cwd=tmp_path, check=True, capture_output=True)
    loads = 0
    for part in sorted(tmp_path.glob("lib.so.*gfx950")):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", part], check=True, capture_output=True, text=True).stdout
        code = []
        for line in text.splitlines():
            line = line.split("//")[0].strip()
            if line:
                code.append(None if line.endswith(":") else line)
        found, n = short_waits(code)
        assert not found, f"{len(found)} of {n} loads in {part.name}, the first: {found[0]}"
        loads += n
    assert loads > 0
