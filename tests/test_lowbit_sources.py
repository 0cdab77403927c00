"""What the sources of the low-bit serving kernels must not do (no GPU needed)."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_05576_b200", "csrc")


def _code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.mark.parametrize("name", ["fp8.cuh", "cache4.cuh", "attn4tile.cuh"])
def test_kernels_that_start_early_read_by_plain_loads(name):
    """Their grids are launched before the kernel that writes their inputs has ended; the read-only path promises that nobody writes
    that memory while a kernel lives, so a compiler may move such a load above the wait."""
    code = _code(name)
    assert "chained_begin()" in code or "chained_wait()" in code
    for word in ("__ldg", "__restrict__", ".nc"):
        assert word not in code, word
