"""Rules of the serving kernels' sources that no run can show to hold, checked on the CPU."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_04105_b200", "csrc")


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))))
def test_no_non_coherent_loads_beside_a_kernel_that_writes(name):
    """A kernel that is launched before its predecessor has ended may read what that one writes.  __ldg and ld.global.nc are defined only for
    memory that is not written while the kernel lives, and a compiler may turn a dereferenced `const T* __restrict__` parameter into one."""
    code = _code(name)
    assert not re.search(r"\b__ldg\b|\bld\.global[.\w:]*\.nc\b", code)
    if name in ("rotary.cu", "kv_cache.cu", "kv_cache.cuh", "tree_attn.cu"):
        assert "__restrict__" not in code
