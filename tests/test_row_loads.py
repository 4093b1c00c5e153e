"""How the kernels over rows of logits read them (host: a look at the source).

A distillation may write its gradient over the logits it reads, within one
launch.  Read-only loads (`ld.global.nc`, `__ldg`) are defined only for memory
that nothing writes while the kernel runs."""
import os
import re

import pytest

from paper_2608_13966_gb300 import build


@pytest.mark.parametrize("name", ["row_stream.cuh", "distill.cuh"])
def test_rows_that_the_launch_may_overwrite_are_not_read_as_constant(name):
    with open(os.path.join(build.CSRC, name)) as f:
        code = re.sub(r"//.*", "", f.read())
    assert not re.search(r"ld\.global\.nc|__ldg\s*\(", code)
