"""What may change from call to call is not read through the read-only path: page tables and shared lists are rewritten while
sequences grow, possibly by the kernel in front, which may still run when a dependent launch begins."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_05787_b200", "csrc")


@pytest.mark.parametrize("name", ["rkv_paged.cu", "rkv_paged_attn.cu", "rkv_prefix.cu", "rkv_pick.cuh"])
def test_only_the_frequencies_are_read_as_constant(name):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    assert all(arg.startswith("p.freqs") for arg in re.findall(r"__ldg\(([^)]*)", text)) and "ld.global.nc" not in text
