"""CPU test of the built library's own code: loads that are written out (inline assembly) keep the wait states that the compiler keeps for the loads it writes itself."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2502_18554_amd import build

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
WAIT_STATES = 5          # between a vector instruction that writes a scalar register and a load that reads it
CARRY = re.compile(r"v_(add_co|addc_co|sub_co|subb_co|subrev_co|subbrev_co|mad_u64|mad_i64|div_scale)")


def registers(text):
    found = set()
    for m in re.finditer(r"\bs(?:(\d+)\b|\[(\d+):(\d+)\])", text):
        found.update([int(m[1])] if m[1] else range(int(m[2]), int(m[3]) + 1))
    return found


def too_early(lines):
    """(function, writer, load) of loads that read a scalar register less than WAIT_STATES after a vector instruction has written it, within straight code; and the number of loads."""
    function, recent, bad, loads = None, [], [], 0
    for line in lines:
        label = re.match(r"[0-9a-f]+ <(.*)>:", line)
        if label:
            function, recent = label[1], []
            continue
        line = line.split("//")[0].strip()
        op, _, operands = line.partition(" ")
        if not op:
            continue
        if op.startswith("buffer_load"):
            loads += 1
            needed, states = registers(operands), 0
            for writes, before in reversed(recent):
                if states >= WAIT_STATES:
                    break
                if writes & needed:
                    bad.append((function, before, line))
                    break
                states += 1 + (int(before.split()[1], 0) if before.startswith("s_nop") else 0)
        writes = set()
        if op.startswith(("v_readfirstlane", "v_readlane", "v_cmp_")):
            writes = registers(operands.split(",")[0])
        elif CARRY.match(op):
            writes = registers(operands.split(",")[1])
        recent = [*recent[-WAIT_STATES:], (writes, line)]
    return bad, loads


def test_the_search_itself():
    early = ["0 <f>:", "  v_readfirstlane_b32 s6, v4", "  s_mov_b32 m0, s20", "  s_nop 0", "  buffer_load_dwordx4 v1, s[4:7], 0 offen lds"]
    assert too_early(early) == ([("f", "v_readfirstlane_b32 s6, v4", "buffer_load_dwordx4 v1, s[4:7], 0 offen lds")], 1)
    for other in ("  s_nop 3", "  s_nop 7"):
        assert too_early([*early[:3], other, early[4]]) == ([], 1)
    assert too_early([early[0], "  v_readfirstlane_b32 s8, v4", *early[2:]]) == ([], 1)


def test_written_out_loads_wait_for_their_buffers(tmp_path):
    if not os.path.exists(build.LIB) or not os.path.exists(OBJDUMP):
        pytest.skip("the library or the disassembler is not there")
    shutil.copy(build.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    parts = sorted(p for p in tmp_path.iterdir() if "gfx950" in p.name)
    assert parts
    loads = 0
    for part in parts:
        with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", part.name], cwd=tmp_path, stdout=subprocess.PIPE, text=True) as p:
            bad, n = too_early(p.stdout)
        assert p.returncode == 0 and not bad, bad[:5]
        loads += n
    assert loads > 1000
