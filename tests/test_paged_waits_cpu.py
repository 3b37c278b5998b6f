"""A wait that runs out ends a kernel with copies under way: they have to land before the CTA gives its shared memory back.  No
test makes such a wait run out, so this reads the source: every way out of a tile loop waits for what was requested."""
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_05787_b200", "csrc", "rkv_paged_attn.cu")


def test_ways_out_of_the_tile_loops_wait_for_their_copies():
    with open(SRC) as f:
        text = f.read()
    out = re.findall(r"!mbar_wait\(bar_(?:full|empty) [^{]*\{(.*?)\n *(?:break|return);", text, re.S)
    assert len(out) == 4                          # a copy warp and the MMA warps, in both kernels
    for block in out:
        assert "RKV_DEV_TIMEOUT" in block and "await_tiles<" in block
