"""Rules of the attention kernels' sources that no healthy run can show to hold, checked on the CPU."""
import re

import pytest

from test_serving_sources import _code


@pytest.mark.parametrize("name", ["attn_fwd.cu", "attn_fwd_2q.cu", "attn_fwd_fp8pv.cu"])
def test_the_last_copies_of_a_block_that_gives_up_are_waited_for(name):
    """Of a barrier's two parities one has always come: a wait for either does not wait."""
    code = _code(name)
    assert not re.search(r"!mbar_try_wait\(([^;]*), 0\) && !mbar_try_wait\(\1, 1\)", code)
    producer = code[code.index("if (warp == 0) {"):code.index("} else if (warp == 1")]
    assert re.search(r"if \(\*abortf\) let_copies_land\(\);\s*__syncwarp\(\);\s*$", producer)
