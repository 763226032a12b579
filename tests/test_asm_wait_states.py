"""CPU test of the memory instructions that the kernels write in inline assembly: between a vector instruction that writes a
scalar register and a memory instruction that reads it the hardware wants five wait states, which the compiler sees to
for its own instructions and not for those in assembly.  So every piece of assembly brings them itself, whatever the compiler
puts in front of it (it may fetch a spilled descriptor with v_readlane just there)."""
import glob
import os
import re
import subprocess

import pytest

from paper_2602_05269_amd import build

STATES = 5
MEMORY = re.compile(r"(buffer|global|flat|scratch)_\w+")
STRING = re.compile(r'"((?:[^"\\]|\\.)*)"')


def _writes_memory_instructions(path):
    text = open(path).read()
    return any(MEMORY.match(line.strip()) for s in STRING.findall(text) for line in s.split("\\n\\t"))


SOURCES = [os.path.basename(p) for p in build.sources() if _writes_memory_instructions(p)]


def test_no_such_assembly_outside_the_sources():
    assert SOURCES                                            # (the search finds the ones that there are)
    for path in glob.glob(os.path.join(build.CSRC, "*.h")):
        assert not _writes_memory_instructions(path), path


@pytest.mark.parametrize("name", SOURCES)
def test_wait_states_in_front_of_memory_instructions(name, tmp_path):
    out = tmp_path / "kernels.s"
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc] + build.HIPCC_FLAGS + ["--cuda-device-only", "-S", os.path.join(build.CSRC, name), "-o", str(out)], check=True,
                   stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    found, states = 0, None                                   # (states: None outside of a piece of assembly)
    for line in out.read_text().splitlines():
        line = line.strip()
        if line == ";;#ASMSTART":
            states = 0
        elif line == ";;#ASMEND":
            states = None
        elif states is not None and line and not line.startswith(";"):
            if MEMORY.match(line):
                found += 1
                assert states >= STATES, f"{line}: {states} wait states in front of it"
            op, *args = line.split()
            assert not op.startswith("v_"), line              # (nothing in it writes a register in the wrong place)
            states += int(args[0], 0) + 1 if op == "s_nop" else 1
    assert found > 0
