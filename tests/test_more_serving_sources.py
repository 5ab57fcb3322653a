"""What the sources of ftint8 and ftdecay have to say to the compiler for their hand-written waits and register writes to hold.
(Where it is missing, today's compiler may still order things well: no result shows it.)"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_02211_amd", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["ftint8.hip", "ftdecay.hip"])
def test_no_memory_operation_moves_behind_a_wait_that_counts_it(name):
    text = source(name)
    waits = [m.start() for m in re.finditer(r"__builtin_amdgcn_s_waitcnt\(", text)]
    assert waits
    for at in waits:
        assert text[:at].rstrip().endswith('asm volatile("" ::: "memory");'), text[max(0, at - 200):at + 40]


@pytest.mark.parametrize("name", ["ftint8.hip", "ftdecay.hip"])
def test_assembly_that_writes_m0_says_so(name):
    found = 0
    for statement in re.findall(r"asm volatile\((?:[^;]|(?<=\\n\\t);)*;", source(name)):
        if re.search(r"s_\w+ m0,", statement):
            found += 1
            assert re.search(r':[^:]*"m0"[^:]*\);$', statement), statement
    assert found


@pytest.mark.parametrize("name", ["ftint8.hip", "ftdecay.hip", "ftsample.hip"])
def test_no_assembly_loads_into_registers(name):
    """(A load in flight would write a register that the compiler takes as written, or as free.)"""
    for statement in re.findall(r'asm(?: volatile)?\(("[^;]*?)\);', source(name), re.S):
        assert not re.search(r"(global|buffer|flat|scratch)_load_(?!lds)", statement) and not re.search(r"ds_(read|load)", statement), statement


@pytest.mark.parametrize("name", ["ftint8.hip", "ftdecay.hip", "ftsample.hip"])
def test_nothing_is_chosen_by_the_environment_or_cleared_by_the_runtime(name):
    text = source(name)
    assert "getenv" not in text and "hipMemset" not in text
