"""Instructions of the products' kernels that want all 32 lanes of a warp together (bar.sync, tcgen05.ld), by reading the sources: in front of
each the warp is brought together, because lanes come there from loops in which each polls by itself, or from what one lane does alone."""
import re

import pytest

from test_bounded_waits import body, source

# .. at once, or with only a choice between them that is the same for all lanes
TOGETHER = r"__syncwarp\(\);\s*$"


def before_each(text, what):
    found = [m.start() for m in re.finditer(what, text)]
    assert found
    return [text[:i].rstrip() for i in found]


def test_named_barrier_of_many_tokens():
    for text in before_each(source("perq_mm_many.cuh"), r'asm volatile\("bar\.sync'):
        assert re.search(TOGETHER, text)


def test_named_barriers_of_rows():
    text = source("perq_quant8.cuh")
    barrier = body(text, "void row_barrier(")
    assert text.count("bar.sync") == barrier.count("bar.sync") > 0
    assert re.search(TOGETHER, barrier[:barrier.index("if (warps == 1)")].rstrip())


@pytest.mark.parametrize("name", ["perq_mm_few.cuh", "perq_mm_many.cuh"])
def test_loads_from_tensor_memory(name):
    for text in before_each(source(name), r"tmem_load16\(tmem|tmem_load16\(from"):
        assert re.search(TOGETHER, text)


@pytest.mark.parametrize("name", ["perq_mm_few.cuh", "perq_mm_many.cuh"])
def test_tensor_memory_is_given_back(name):
    """(tcgen05.dealloc, also where nothing was split and the cluster's barrier, which is for single threads, is the last thing before it)"""
    text = source(name)
    end = text[:text.index("tcgen05.dealloc")]
    assert re.search(r"__syncwarp\(\);\s*if \(warp == 1\) \{\s*tmem_fence_after\(\);\s*asm volatile\(\"$", end)
