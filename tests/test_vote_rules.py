"""Lanes of a warp whose bounded waits run out apart must not part, checked in the source."""
import os
import re

import pytest

from test_launch_rules import CSRC, _strip_comments


@pytest.mark.parametrize("name,loop", [("mwu_grouped.cu", "for (int b0 = c0; b0 < c1; b0 += BL)"),
                                       ("mwu_gemm3.cu", "const unsigned live = lv[ks];\n                if (!live) continue;\n                if (!mbar_wait_spin(")])
def test_lanes_that_leave_the_loop_of_the_mmas_need_no_others_in_it(name, loop):
    # Every lane waits for itself and may leave the loop alone.  A vote, an election or a warp barrier inside it, which name all 32
    # lanes, would keep those that go on waiting for the ones that left.
    text = _strip_comments(open(os.path.join(CSRC, name)).read())
    assert text.count(loop) == 1
    start = text.index(loop)
    body = text[start:text.index("__all_sync(0xffffffffu, ok)", start)]
    assert "mbar_wait_spin(" in body and "if (leader)" in body
    assert not re.search(r"elect_one|_sync\(|__syncwarp|warp_wait", body)
    assert re.search(r"const bool leader = elect_one\(\);", text[:start])
