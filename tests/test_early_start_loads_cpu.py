"""Kernels that start while the one before them may still run read a caller's memory by ordinary or L2 loads.

The read-only path is for memory that nobody writes while the kernel exists.  A kernel launched with programmatic dependence exists before the one
in front of it has ended, and its wait orders ordinary loads, not that path.  Nothing here can make a stale read happen on demand, so the
sources are read.  (The 8-bit float products are not among these files: they read the scales of weights so, which are written before
such a product is launched at all.)
"""
from __future__ import annotations

import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2410_07505_b200", "csrc")
FILES = ("cq_prompt.cu", "cq_rotate.cu", "cq_adapter.cu", "cq_adapter.cuh", "cq_adapter_tiles.cu", "cq_kv.cu", "cq_kv.cuh", "cq_kv_attend.cu")


@pytest.mark.parametrize("name", FILES)
def test_no_read_only_loads(name):
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert not re.search(r"__ldg\s*\(|\bld_nc\s*\(|ld\.global(\.\w+)*\.nc", text)
    assert "__restrict__" not in text                           # (which lets the compiler choose that path by itself)
    if name.endswith(".cu"):
        assert "griddepcontrol.wait" in text
