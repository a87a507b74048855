"""Barriers written as builtins: the compiler takes them for touching no memory, so the sources have to keep accesses on their side."""
import glob
import os
import re

import pytest

import paper_1908_06077_amd as nuq

CSRC = os.path.join(os.path.dirname(os.path.abspath(nuq.__file__)), "csrc")
CLOBBER = 'asm volatile("" ::: "memory");'
BARRIER = "__builtin_amdgcn_s_barrier();"


def statements(text):
    return [s.strip() for s in re.split(r"[;{}]", re.sub(r"//[^\n]*", "", text)) if s.strip()]


@pytest.mark.parametrize("name", sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*.h*"))))
def test_accesses_stay_on_their_side(name):
    """Between a clobber and a barrier there are waits alone, and a clobber is the first thing behind it."""
    with open(os.path.join(CSRC, name)) as f:
        parts = f.read().split(BARRIER)
    for before, after in zip(parts, parts[1:]):
        assert CLOBBER in before
        between = statements(before[before.rindex(CLOBBER) + len(CLOBBER):])
        assert all(re.fullmatch(r"(else )?(if \(.*\)\s*|else\s*)?__builtin_amdgcn_s_waitcnt\(.*\)", s, re.S) for s in between), between
        assert re.sub(r"//[^\n]*", "", after).lstrip().startswith(CLOBBER)


def test_there_are_such_barriers():
    found = 0
    for p in glob.glob(os.path.join(CSRC, "*.h*")):
        with open(p) as f:
            found += f.read().count(BARRIER)
    assert found >= 2
