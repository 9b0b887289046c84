"""What the kernels' inline assembly tells the compiler."""
import glob
import os
import re

import pytest

from paper_2603_27138_amd import build

SOURCES = sorted(glob.glob(os.path.join(build.CSRC, "*.h*")))


def _statements(text):
    """The asm statements of a source, parentheses and strings matched."""
    for start in re.finditer(r"\basm\s+volatile\s*\(", text):
        depth, quoted, at = 1, False, start.end()
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            at += 1
        yield text[start.start():at]


def _writes_m0(statement):
    return re.search(r"\bs_\w+ m0\b", statement) is not None


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_m0_is_named_where_it_is_written(path):
    """The compiler may keep a value of its own in m0 across a statement that does not say it writes there."""
    with open(path) as f:
        for s in _statements(f.read()):
            if _writes_m0(s):
                assert s.rstrip(") ").endswith('"m0"') or '"m0",' in s, s


def test_the_search_finds_what_it_is_for():
    text = 'a(); asm volatile("s_mov_b32 m0, %1\\n\\tx (" ::"s"(r), "s"(to) : "memory"); asm volatile("s_barrier");'
    found = list(_statements(text))
    assert len(found) == 2 and _writes_m0(found[0]) and not _writes_m0(found[1])
    assert any(_writes_m0(s) for path in SOURCES for s in _statements(open(path).read()))


def _waits_in_front_of_the_first_load(statement):
    """Wait states: one for each instruction, n + 1 for s_nop n."""
    code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', statement.split("::")[0]))
    waits = 0
    for line in code.split("\\n\\t"):
        if re.match(r"(buffer|global|flat)_load", line):
            return waits
        nop = re.match(r"s_nop (\d+)", line)
        waits += int(nop[1]) + 1 if nop else 1
    return None


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_scalar_operands_of_loads_are_waited_for(path):
    """A vector instruction that writes a scalar register needs five wait states in front of a load that reads it.  The compiler keeps them
    between its own instructions; into a statement it does not look."""
    with open(path) as f:
        for s in _statements(f.read()):
            waits = _waits_in_front_of_the_first_load(s)
            if waits is not None and '"s"(' in s:
                assert waits >= 5, s


def test_wait_states_are_counted():
    assert _waits_in_front_of_the_first_load(r'asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tbuffer_load_dword %2" ::"s"(r))') == 5
    assert _waits_in_front_of_the_first_load('asm volatile("s_barrier" ::)') is None
