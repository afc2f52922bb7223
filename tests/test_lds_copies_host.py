"""Copies from memory straight into LDS that are written as assembly (no GPU): what the hardware wants
between their instructions, and the compiler does not add inside an asm block, is there.

A load to LDS takes its LDS address from m0.  After a scalar write of m0 it needs one wait state, that
is an s_nop or an independent instruction between the two; between instructions of its own the compiler
for gfx950 puts an s_nop there."""
import os
import re

import pytest

from paper_2606_03077_amd import build

SOURCES = [s for s in build.SOURCES if s.endswith(".hip")]


def blocks(text):
    """The instructions of each asm block, one string a line."""
    for m in re.finditer(r"\basm\s+volatile\s*\(\s*((?:\"(?:[^\"\\]|\\.)*\"\s*)+)", text):
        code = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", m.group(1)))
        yield [line.strip() for line in re.split(r"\\n|;", code.replace("\\t", " ")) if line.strip()]


def missing_waits(text):
    """Blocks in which a load to LDS comes right behind a write of m0, or first, behind what may write it."""
    bad = []
    for code in blocks(text):
        for i, line in enumerate(code):
            if re.match(r"(global|buffer|scratch)_load\w*_lds|buffer_load\w*.*\blds\b", line):
                if i == 0 or re.match(r"s_\w+\s+m0\b", code[i - 1]):
                    bad.append(code)
    return bad


def test_the_scan_sees_a_missing_wait():
    near = r'asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off" : : "s"(d), "v"(s) : "m0");'
    assert len(missing_waits(near)) == 1
    assert not missing_waits(near.replace(r"\tglobal", r"\ts_nop 0\n\tglobal"))
    assert len(missing_waits('asm volatile("buffer_load_dword %0, s[0:3], 0 offen lds" : : "v"(x));')) == 1


@pytest.mark.parametrize("source", SOURCES)
def test_loads_to_lds_wait_for_m0(source):
    with open(os.path.join(build.CSRC, source)) as f:
        text = f.read()
    assert not missing_waits(text)
    # The scan looks at every block that there is.
    assert len(list(blocks(text))) == len(re.findall(r"\basm\s+volatile", text))


def test_there_are_such_copies():
    found = 0
    for source in SOURCES:
        with open(os.path.join(build.CSRC, source)) as f:
            found += sum(any("_lds_" in line for line in code) for code in blocks(f.read()))
    assert found >= 3
