"""Waits that the hardware does not make by itself and the compiler does not put into inline assembly, read out of the sources: between a write of m0 and a load into the LDS that goes by it, one;
between a scalar that comes out of a vector register and a load by that base, five (the compiler may put the former right before the assembly)."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_01815_amd", "csrc")
SOURCES = sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h")))


def loads_into_the_lds(text):
    """[(instructions from the write of m0 to the load, between them; the load's last operand)] of every piece of inline assembly with such a load."""
    found = []
    for piece in re.findall(r'asm(?:\s+volatile)?\s*\(\s*((?:"(?:[^"\\]|\\.)*"\s*)+)', text):
        lines = [x.strip() for x in "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', piece)).replace("\\t", " ").split("\\n")]
        for i, line in enumerate(lines):
            if re.match(r"(global|buffer)_load_lds|(global|buffer)_load.* lds$", line):
                wrote = [j for j in range(i) if re.match(r"s_mov_b32 m0,", lines[j])]
                found.append((lines[wrote[-1] + 1:i] if wrote else None, line.split(",")[-1].split()[0]))
    return found


def waits(lines):
    return sum(int(m.group(1)) + 1 if (m := re.match(r"s_nop (\d+)", x)) else 1 for x in lines)


def test_the_reader_finds_loads():
    text = 'asm volatile("s_mov_b32 m0, %0\\n\\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to)); asm("s_mov_b32 m0, %1\\n\\ts_nop 2\\n\\t" "global_load_lds_dword %0, off nt" : );'
    assert loads_into_the_lds(text) == [([], "%2"), (["s_nop 2"], "off")] and waits(["s_nop 2", "s_mov_b32 s0, s1"]) == 4
    assert sum(len(loads_into_the_lds(open(os.path.join(CSRC, f)).read())) for f in SOURCES) >= 5


@pytest.mark.parametrize("source", SOURCES)
def test_loads_into_the_lds_wait_for_their_address(source):
    for between, _ in loads_into_the_lds(open(os.path.join(CSRC, source)).read()):
        assert between is not None and waits(between) >= 1, source


@pytest.mark.parametrize("source", SOURCES)
def test_loads_into_the_lds_wait_for_their_base(source):
    for between, last in loads_into_the_lds(open(os.path.join(CSRC, source)).read()):
        assert last == "off" or waits(between) + 1 >= 5, source              # (the write of m0 is one)
