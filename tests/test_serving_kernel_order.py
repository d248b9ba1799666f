"""Orders within the FFN step's kernel on which progress depends and which a run does not show: read from the source."""
import os
import re

import pytest

from paper_2506_18145_b200 import build as rbuild

from test_kernel_order import kernels


@pytest.fixture(scope="module")
def body():
    body, = [k for k in kernels(os.path.join(rbuild.CSRC, "rom_ffn_step.cu")) if "tcgen05.alloc" in k]
    return body


def test_the_successor_comes_in_behind_the_tensor_memory_of_the_block(body):
    """The warp that allocates lets in, behind its allocation; the others may be ahead of it."""
    alloc = re.search(r"if \(warp == (\d+)\) \{\s*asm volatile\(\"tcgen05\.alloc", body)
    first = re.search(r"pdl_trigger\(\)", body)
    assert alloc.start() < first.start() < body.index("__syncthreads();\n  tc_fence_after();")
    assert f"if (warp == {alloc.group(1)}) pdl_trigger();" in body[first.start() - 20:first.end() + 1]


@pytest.mark.parametrize("what", [r'asm volatile\("bar\.sync', r"bar\.red", r"tmem_ld32_issue\(taddr \+ c0", r"tc_fence_after\(\);\s*asm volatile\(\"tcgen05\.dealloc"])
def test_warps_meet_before_aligned_instructions(body, what):
    """The statement before is the one that brings the lanes of a warp together."""
    found = list(re.finditer(what, body))
    assert found
    for m in found:
        before = body[:body.rindex("asm volatile", 0, m.end())] if "bar" in what else body[:m.start()]
        assert before.rstrip().endswith("__syncwarp();")
