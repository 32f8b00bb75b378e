"""An order that kernels keep in their source: tensor memory before the next kernel may come up."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34045_gb300", "csrc")


def kernels():
    """(file, name, body) of every kernel that allocates tensor memory."""
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        for m in re.finditer(r"__global__[^;{]*?\b(\w+_kernel)\s*\([^;{]*\{", text):
            depth, end = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[end], 0)
                end += 1
            body = text[m.end():end]
            if "tmem_alloc(" in body:
                yield pytest.param(body, id=f"{os.path.basename(path)}:{m.group(1)}")


def test_kernels_are_found():
    assert len(list(kernels())) >= 3


@pytest.mark.parametrize("body", list(kernels()))
def test_tensor_memory_is_taken_before_dependents_are_let_in(body):
    """A dependent kernel's block that is resident before this kernel's block has allocated may take the tensor memory and then
    wait for this grid's end, which waits for the tensor memory.  All of the block's threads have to know that it is allocated."""
    alloc, launch = body.index("tmem_alloc("), body.index("pdl_launch_dependents()")
    assert alloc < launch
    assert "__syncthreads()" in body[alloc:launch]
