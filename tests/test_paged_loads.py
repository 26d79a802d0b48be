"""The paged-cache kernels are launched while the kernel before them in the stream
may still run (programmatic stream serialisation) and read what it writes: lengths,
page tables, exponents, rotated queries. A read-only (non-coherent) load is defined
only for memory that nothing writes during its kernel's whole life, so these sources
hold none. A wrong value would be a race, which no run shows: the sources are read."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_23144_gb300", "csrc")
EARLY = [f for f in sorted(os.listdir(CSRC)) if f.endswith((".cu", ".cuh"))
         and re.search(r"\blaunch_next\(|\bwait_for_previous\(", open(os.path.join(CSRC, f)).read())]


def test_the_kernels_launched_early_are_found():
    assert EARLY == ["kv_append.cu", "kv_paged.cuh", "paged_attn.cu", "paged_tiles.cu"]


@pytest.mark.parametrize("name", EARLY)
def test_kernels_launched_early_have_no_read_only_loads(name):
    code = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    # the intrinsic, its PTX form, and the qualifier that lets the compiler choose it
    assert not re.search(r"\b__ldg\b|\bld\.global(\.\w+)*\.nc\b|\b__restrict__\b", code)
