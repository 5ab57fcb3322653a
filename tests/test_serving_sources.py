"""What the serving kernels' sources have to say to the compiler for their hand-written waits and register writes to hold.
(Where it is missing, today's compiler may still order things well: no result shows it.)"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_02211_amd", "csrc")


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["ftprompt.hip", "ftcache.hip"])
def test_no_memory_operation_moves_behind_a_wait_that_counts_it(name):
    """The wait instruction touches no memory as far as the compiler knows: what has to be complete behind it is held before it by an empty
    statement that touches all memory."""
    text = source(name)
    waits = [m.start() for m in re.finditer(r"__builtin_amdgcn_s_waitcnt\(", text)]
    assert waits
    for at in waits:
        assert text[:at].rstrip().endswith('asm volatile("" ::: "memory");'), text[max(0, at - 200):at + 40]


@pytest.mark.parametrize("name", ["ftprompt.hip", "ftcache.hip", "ftserve_device.h"])
def test_assembly_that_writes_m0_says_so(name):
    for statement in re.findall(r"asm volatile\((?:[^;]|(?<=\\n\\t);)*;", source(name)):
        if re.search(r"s_\w+ m0,", statement):
            assert re.search(r':[^:]*"m0"[^:]*\);$', statement), statement
