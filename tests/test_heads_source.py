"""What the sources of the multi-class head's kernels have to say for themselves, because no run shows it, and the knob of its tiles."""
import os
import re

import pytest

import paper_2008_03433_amd as tron

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2008_03433_amd", "csrc")
FENCE = 'asm volatile("" ::: "memory");'


def test_raw_barriers_lie_between_compiler_barriers():
    """The barrier instruction alone orders nothing for the compiler, which may move accesses of LDS across it."""
    found = 0
    for name in ("head_norm.hip", "head_linear.hip", "head_distill.hip", "head_util.h"):
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        lines = [line.strip() for line in text.splitlines() if line.strip()]
        for i, line in enumerate(lines):
            if "__builtin_amdgcn_s_barrier()" in line:
                found += 1
                assert lines[i - 1].startswith("__builtin_amdgcn_s_waitcnt("), (name, line)
                assert lines[i - 2] == FENCE and lines[i + 1] == FENCE, (name, lines[i - 2:i + 2])
    assert found


def test_the_knob_of_the_tiles():
    lib, sizes = tron.load_library(), {}
    try:
        for side in (128, 256):
            tron.tron_tuning_set("linear_tile", side)
            sizes[side] = lib.tron_linear_work(700, 600, 8192, 1)
            assert sizes[side] > 0   # the inner index is cut in either
        assert sizes[128] != sizes[256]
        for wrong in (-1, 64, 512):
            with pytest.raises(tron.TronError):
                tron.tron_tuning_set("linear_tile", wrong)
    finally:
        tron.tron_tuning_set("linear_tile", 0)
    assert lib.tron_linear_work(700, 600, 8192, 1) in sizes.values()
