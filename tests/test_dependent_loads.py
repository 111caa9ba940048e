"""Kernels that may start before the one they depend on has finished (`griddepcontrol.wait`) read nothing through the read-only
path: such a load counts as invariant, so it may be moved above the wait, and wants data that nobody writes while the kernel lives."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_17353_b200", "csrc")
READ_ONLY = re.compile(r"\b__ldg\s*\(|\bload_scale\s*\(|ld\.global\.nc")


@pytest.mark.parametrize("name", ["linear_loss.cu"])
def test_no_read_only_loads(name):
    """Every kernel of the file is such a one, so the whole file is looked at, its helpers too."""
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    kernels = code.split("__global__")[1:]
    assert len(kernels) >= 6 and all("griddepcontrol.wait" in k for k in kernels)
    assert not [line.strip() for line in code.split("\n") if READ_ONLY.search(line)]
