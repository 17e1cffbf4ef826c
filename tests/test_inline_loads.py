"""LDS loads in inline assembly of the tree attention's kernels.  The compiler takes a
statement's registers as written when the statement is, so a load that is waited for later could
be copied, spilled or have its registers reused before its value arrives: every
statement that loads has to wait for its loads itself."""
import os
import re

import pytest

from paper_2604_20919_amd import build


def statements(source):
    """The instructions of every inline assembly statement of a source, in order."""
    out = []
    for m in re.finditer(r"\basm\s*(?:volatile)?\s*\(", source):
        text = re.match(r'(?:\s*"(?:[^"\\]|\\.)*")+', source[m.end():])
        if text:
            parts = re.findall(r'"((?:[^"\\]|\\.)*)"', text.group(0))
            out.append([i.strip() for i in re.split(r"\\n|\\t|\n|;", "".join(parts)) if i.strip()])
    return out


def unwaited(instructions):
    """The loads of a statement that its own waits do not cover (LDS operations return in order)."""
    flight = []
    for i in instructions:
        if re.match(r"(ds|buffer|global|flat|scratch|s)_(read|load|gather)", i) and not i.endswith(" lds"):
            flight.append(i)
        elif i.startswith("s_waitcnt"):
            left = re.search(r"lgkmcnt\((\d+)\)", i)
            if left:
                flight = flight[len(flight) - int(left.group(1)):] if int(left.group(1)) else []
    return flight


def test_the_reader():
    waits = 'asm volatile("ds_read_b128 %0, %1\\n\\t"\n  "s_waitcnt lgkmcnt(0)" : "=&v"(a) : "v"(b));'
    late = 'asm volatile("ds_read_b128 %0, %2\\n\\tds_read_b128 %1, %2 offset:1024" : "=&v"(a), "=&v"(c) : "v"(b));'
    assert statements(waits) == [["ds_read_b128 %0, %1", "s_waitcnt lgkmcnt(0)"]] and unwaited(statements(waits)[0]) == []
    assert len(unwaited(statements(late)[0])) == 2
    assert unwaited(["ds_read_b32 %0, %1", "ds_read_b32 %2, %1", "s_waitcnt lgkmcnt(1)"]) == ["ds_read_b32 %2, %1"]
    assert unwaited(["s_waitcnt lgkmcnt(0)", "ds_read_b32 %0, %1"]) and unwaited(["global_load_dword %0, %1, off", "s_nop 0"])


@pytest.mark.parametrize("name", ["k_tree.hip"])
def test_every_statement_waits_for_its_loads(name):
    with open(os.path.join(build.CSRC, name)) as f:
        found = statements(f.read())
    assert any(i.startswith("ds_read") for s in found for i in s)
    assert [s for s in found if unwaited(s)] == []
