"""How kernels that start while the grid before them still runs read memory (host: a look at
the source).

A programmatic dependent waits for that grid, which may still be writing what it is going to
read.  Read-only loads (`ld.global.nc`, `__ldg`) are defined only for memory that nothing
writes while the kernel runs, from its start and not from that wait on, and the compiler may
move them above it."""
import glob
import os
import re

import pytest

from paper_2608_13966_gb300 import build

SOURCES = {os.path.basename(p): open(p).read() for p in glob.glob(os.path.join(build.CSRC, "*.cuh"))}
DEPENDENTS = sorted(n for n, s in SOURCES.items() if "wait_for_previous_grid();" in s)


def included(name, seen=None):
    """A source and those that it includes."""
    seen = {} if seen is None else seen
    if name not in seen and name in SOURCES:
        seen[name] = SOURCES[name]
        for other in re.findall(r'#include "([^"]+)"', SOURCES[name]):
            included(other, seen)
    return seen


def test_there_are_dependents():
    assert {"linear.cuh", "linear_one.cuh", "linear_grad.cuh", "distill.cuh", "top_logits.cuh"} <= set(DEPENDENTS)


@pytest.mark.parametrize("name", DEPENDENTS)
def test_dependents_have_no_read_only_loads(name):
    for part, text in included(name).items():
        code = re.sub(r"//.*", "", text)
        assert not re.search(r"ld\.global\.nc|__ldg\s*\(|__restrict__", code), part
