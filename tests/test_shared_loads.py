"""Loads straight to shared memory are written out, so that the compiler does not see them: what it would keep between them and the instructions
before them has to stand there.  Read from the code of the library that is built here.

A load that reads a scalar register wants five wait states behind a vector instruction that has written it (a lane read first, or a spilled value read back), and
one behind the write of m0.  An instruction is one state, `s_nop n` n + 1.  Either the states are there, or the load's base is a scalar instruction's, which waits for a
vector instruction's write by itself, and no vector instruction in these five states writes the same register.
"""
import os
import re
import struct
import subprocess

import pytest

from test_register_budget import LIB

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
pytestmark = pytest.mark.skipif(not os.path.exists(LIB) or not os.path.exists(OBJDUMP), reason="the library is not built, or there is nothing to list it with")


def code_objects(path):
    """The AMDGPU code objects inside the library: whole ELF files, whose section headers come last."""
    data = open(path, "rb").read()
    for m in re.finditer(rb"\x7fELF\x02\x01\x01", data):
        at = m.start()
        machine, = struct.unpack_from("<H", data, at + 18)
        if machine == 224:
            headers, = struct.unpack_from("<Q", data, at + 40)
            size, count = struct.unpack_from("<HH", data, at + 58)
            yield data[at:at + headers + size * count]


def numbers(operand):
    """Scalar registers that an operand names."""
    m = re.fullmatch(r"s(\d+)|s\[(\d+):(\d+)\]", operand.strip())
    return set(range(int(m.group(1) or m.group(2)), int(m.group(1) or m.group(3)) + 1)) if m else set()


def test_wait_states_before_loads_to_shared_memory(tmp_path):
    loads = 0
    for i, code in enumerate(code_objects(LIB)):
        if b"k_prompt_" not in code:
            continue
        at = tmp_path / f"{i}.co"
        at.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--mcpu=gfx950", str(at)], capture_output=True, text=True, check=True).stdout
        lines = [x.split("//")[0].strip() for x in listing.splitlines()]
        lines = [x for x in lines if x and not x.endswith(">:")]
        for k, line in enumerate(lines):
            if not re.match(r"(global|buffer)_load_(lds_|.* lds$)", line):
                continue
            loads += 1
            base = numbers(line.split(",")[-1].split()[0])
            assert len(base) == 2, line
            states, back, moved, m0 = 0, k - 1, False, None
            while states < 5:
                name, _, operands = lines[back].partition(" ")
                writes = numbers(operands.split(",")[0]) if name != "s_nop" else set()
                assert not name.startswith(("s_branch", "s_cbranch")) or m0, lines[back:k + 1]
                if name.startswith("v_"):
                    assert not writes & base, lines[back:k + 1]
                if operands.startswith("m0,") and m0 is None:
                    m0 = states
                moved |= name == "s_mov_b64" and writes == base
                states += int(operands) + 1 if name == "s_nop" else 1
                back -= 1
            assert m0 and (moved or all(x.startswith("s_") for x in lines[back + 1:k])), lines[back:k + 1]
    assert loads >= 100
