"""The kernels' inline assembly holds no instruction that reads or writes registers.

The compiler keeps the distances that the hardware asks for between instructions (an
MFMA's results need up to 18 wait states before a vector instruction reads them), but
it does not look into inline assembly: a vector instruction there could read what is
not written yet.  Empty statements (they order memory accesses and hold values) and
waits on counters are all that the sources use."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_21706_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.h")) + glob.glob(os.path.join(CSRC, "*.hip")))
STATEMENT = re.compile(r'\b(?:asm|__asm|__asm__)\b\s*(?:(?:volatile|__volatile__|goto|inline)\b\s*)*\(\s*((?:"(?:[^"\\]|\\.)*"\s*)*)')


def templates(text):
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    return ["".join(re.findall(r'"((?:[^"\\]|\\.)*)"', m.group(1))) for m in STATEMENT.finditer(text)]


def allowed(template):
    return all(not line.strip() or line.strip().startswith("s_waitcnt ")
               for line in re.split(r"\\n|;", template))


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_no_instruction_on_registers(path):
    assert [t for t in templates(open(path).read()) if not allowed(t)] == []


def test_the_search_finds_statements():
    text = 'asm("v_max3_f32 %0, %1" : "=v"(a) : "v"(b)); asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); asm volatile("" : "+v"(x));'
    assert [allowed(t) for t in templates(text)] == [False, True, True]
    assert sum(len(templates(open(path).read())) for path in SOURCES) > 10
