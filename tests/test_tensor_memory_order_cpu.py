"""A kernel lets the next one begin only when it has its columns of tensor memory.

An allocation waits, without a limit, until there are columns enough.  A kernel that is launched with programmatic dependence may come
to an SM as soon as every block of the one before it has said `launch_dependents`; had one of those not allocated yet, the later
kernel could take the columns, and each would wait for the other's end for good.  That cannot be shown on a GPU without hanging it, so
this reads the sources: the instruction stands behind the barrier that follows the allocation.
"""
from __future__ import annotations

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_07505_b200", "csrc")


def kernels(text):
    """(name, body) of each __global__ function; a body ends with the first brace in column 0."""
    for m in re.finditer(r"^__global__ void\s+(?:__launch_bounds__\([^\n]*\)\s+)?(\w+)\(", text, re.M):
        yield m.group(1), text[m.end():text.index("\n}", m.end())]


def uncommented(path):
    with open(path) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def order_of(body):
    """Places of the last allocation, of the block's first barrier behind it, and of the first release of dependents (None: there is none)."""
    allocated = body.rfind("tmem_alloc(")
    released = body.find("griddepcontrol.launch_dependents")
    return allocated, body.find("__syncthreads();", allocated), None if released < 0 else released


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu"))), ids=os.path.basename)
def test_dependents_begin_behind_the_allocation(path):
    for name, body in kernels(uncommented(path)):
        if "tmem_alloc(" not in body:
            continue
        allocated, barrier, released = order_of(body)
        assert 0 < allocated < barrier, name
        assert released is None or barrier < released, name


def test_the_kernels_that_allocate_are_seen():
    seen = {name for path in glob.glob(os.path.join(CSRC, "*.cu")) for name, body in kernels(uncommented(path)) if "tmem_alloc(" in body}
    assert seen == {"k12_product", "k13_product_few", "k22_prompt", "k27_adapter_in_tiles", "k28_adapter_out_tiles"}
    good = 'if (warp == 1) tmem_alloc(&s, 512);\n__syncthreads();\nasm volatile("griddepcontrol.launch_dependents;");'
    allocated, barrier, released = order_of(good)
    assert allocated < barrier < released
    allocated, barrier, released = order_of('asm volatile("griddepcontrol.launch_dependents;");\n' + good)
    assert released < allocated
