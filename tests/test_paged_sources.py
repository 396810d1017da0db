"""Rules of the sources of attention over a cache that no healthy run can show to hold, checked on the CPU."""
import re

import pytest

from test_serving_sources import _code


@pytest.mark.parametrize("name", ["tree_attn.cu", "paged_attn.cu"])
def test_nothing_is_brought_into_a_stage_that_has_not_become_free(name):
    """A wait that sees the abort word returns although its phase has not come, and after that those who read stages free them unread.  An arrival at a barrier
    that still expects bytes is one too many, and a copy into its stage would lie over one under way: between a wait for a stage and the arrival that
    announces a copy, the abort word is looked at and ends the bringing, for the whole warp alike."""
    code = _code(name)
    places = [m.start() for m in re.finditer(r"\bmbar_arrive_expect_tx\(", code)]
    assert places
    for at in places:
        wait = list(re.finditer(r"\bwait(_phase<CALL>)?\([^;]*;", code[:at]))[-1]
        between = code[wait.end():at]
        assert re.search(r"given_up\(abort_at\)", between) and re.search(r"\b(break|return false);", between), between
    # nobody goes on as if a part had been brought
    for m in re.finditer(r"[^;{}]*\bpages\.bring\(", code):
        assert "!pages.bring(" in m.group(), m.group()
    body = re.search(r"\bbool given_up\(.*?\n}", _code("cache_attn.cuh"), re.S).group()
    assert "ld.volatile.shared" in body and "return __shfl_sync(0xffffffffu, gone, 0)" in body          # the word itself, one answer for the warp


def test_the_last_copies_are_waited_for_whatever_the_abort_word_says():
    """A block whose copies are still under way must not end: after a wait has run out, too, and for a limited time."""
    shared = _code("cache_attn.cuh")
    body = re.search(r"\bvoid drain\(.*?\n}", shared, re.S).group()
    assert "spin < (1 << 13) && !mbar_try_wait(" in body and "abort" not in body and "wait_phase" not in body
    for name, kernels in (("tree_attn.cu", 2), ("paged_attn.cu", 1)):
        code = _code(name)
        # by the warp that has brought them, or, where every warp brings some, by the block when it has given up
        drains = len(re.findall(r"\bdrain\([^;]*RING_FULL\), (?:pages\.i|parts)\);", code))
        drains += len(re.findall(r"if \(threadIdx\.x < 2 \* C::kStages\)\s*for \(int spin = 0; spin < \(1 << 10\) && !mbar_try_wait\(full", code))
        assert drains == kernels


@pytest.mark.parametrize("name", ["cache_attn.cuh", "paged_attn.cu", "pages.cu"])
def test_no_pointer_is_said_to_be_the_only_one(name):
    """As of the other serving kernels: a load through `const T* __restrict__` may become one that is not coherent."""
    assert "__restrict__" not in _code(name)
