"""What the sources of kernels in clusters and on the tensor cores have to say, because no run would show it for certain."""
import os
import re

import pytest

from paper_1803_04209_b200 import build


def _source(name: str) -> str:
    with open(os.path.join(build.CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


# A barrier of the cluster, or of some of a CTA's warps, takes whole warps (.aligned), and lanes leave a branch when they like.
@pytest.mark.parametrize("name", ["tcgen05.cuh", "int8_tc.cuh", "kernels_model.cuh", "fit.cuh"])
def test_lanes_meet_before_a_barrier_that_takes_whole_warps(name):
    source = _source(name)
    found = list(re.finditer(r'asm volatile\("(?:barrier\.cluster\.arrive[^"]*\.aligned|bar\.sync)[^"]*"', source))
    assert found
    for m in found:
        before = source[: m.start()].rstrip()
        assert before.endswith("__syncwarp();"), source[m.start(): m.end()]


def _body(source: str, kernel: str) -> str:
    at = source.index("{", source.index(kernel + "("))
    depth, i = 1, at + 1
    while depth:
        depth += {"{": 1, "}": -1}.get(source[i], 0)
        i += 1
    return source[at: i]


# All tcgen05 instructions of a kernel have one group size: those of the kernels on pairs of SMs have two, their tensor memory included.
@pytest.mark.parametrize("name,kernel", [("int8_tc.cuh", "k_product_pair"), ("emit_tc2.cuh", "k_emit_tc2")])
def test_kernels_on_pairs_name_one_group_size(name, kernel):
    body = _body(_source(name), kernel)
    assert "cta_group::1" not in body and "umma_commit(" not in body and "umma_s8(" not in body
    for helper in ("tmem_alloc_pair", "tmem_free_pair", "umma_commit_pair"):
        assert helper in body and "cta_group::1" not in _body(_source("tcgen05.cuh"), "void " + helper)
