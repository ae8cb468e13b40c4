"""Rules of the attention kernels over the cache that a run on a GPU must not be made to break.  Checked on the source text (no GPU)."""
import os
import re

import pytest

import paper_2603_15965_b200 as M

CSRC = os.path.join(os.path.dirname(M.__file__), "csrc")


def text(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_every_kernel_that_takes_tmem_is_looked_at():
    users = {f for f in os.listdir(CSRC) if f.endswith(".cu") and "take_tmem(" in text(f)}
    assert users == {"kv_attend_stream.cu", "kv_attend_tiles.cu"}


@pytest.mark.parametrize("name", ["kv_attend_stream.cu", "kv_attend_tiles.cu"])
def test_tmem_is_taken_after_the_wait_and_before_the_successor_may_start(name):
    """As for the other chained kernels: the allocation has no limit, so a CTA must not hold columns that its predecessor still waits for, and
    must have its own before a successor can take them; nothing from another kernel is read before the wait."""
    code = text(name)
    start = re.search(r"__global__ void[^;{]*\battend_(stream|tiles)_kernel\(", code).end()
    code = code[start:code.index("\n}\n", start)]
    wait, alloc = code.index("grid_dependency_wait()"), code.index("take_tmem(")
    barrier = code.index("__syncthreads()", alloc)
    trigger = code.index("grid_dependency_trigger()")
    assert wait < alloc < barrier < trigger
    assert not re.search(r"ld_dependent|sequence_of|cut_shares|ld128_rw", code[:wait])
    assert code.index("tmem_dealloc(") > code.rindex("__syncthreads()")


@pytest.mark.parametrize("name", ["kv_attend_stream.cu", "kv_attend_tiles.cu", "kv_attend.cuh"])
def test_every_wait_has_a_limit(name):
    """Barriers in shared memory are waited for by wait_bar, or in a loop that looks at the clock."""
    code = text(name)
    for m in re.finditer(r"while \(!mbar_try_wait\([^;]*\)\)\s*([^;]*;)", code):
        assert "kTimeoutCycles" in m.group(1) and "break" in m.group(1)
    assert len(re.findall(r"mbar_try_wait\(", code)) == len(re.findall(r"while \(!mbar_try_wait\(", code))
