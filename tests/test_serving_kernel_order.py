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
