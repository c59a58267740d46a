"""What the sources of the layer operators' tensor-core kernels have to say, because no run would show it for certain."""
import os
import re

import pytest

from paper_1803_04209_b200 import build


def _source(name: str) -> str:
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


# A barrier of the cluster, or of some of a CTA's warps, takes whole warps (.aligned), and lanes leave a branch when they like.
@pytest.mark.parametrize("name", ["tcgen05.cuh", "int8_tc.cuh"])
def test_lanes_meet_before_a_barrier_that_takes_whole_warps(name):
    source = _source(name)
    found = list(re.finditer(r'asm volatile\("(?:barrier\.cluster\.arrive[^"]*\.aligned|bar\.sync)[^"]*"', source))
    assert found
    for m in found:
        before = source[: m.start()].rstrip()
        assert before.endswith("__syncwarp();"), source[m.start(): m.end()]
