"""A ring slot that plain accesses of a warp touched goes back to the copy engine, checked in the source."""
import os
import re

from test_launch_rules import CSRC, _strip_comments


def test_a_slot_goes_back_behind_all_lanes():
    # One lane gives the slot back for its warp, and the next TMA load into it is ordered behind the other lanes' plain accesses by
    # nothing but a proxy fence behind the writes, whichever way the box leaves, and a warp barrier behind the reads.
    text = _strip_comments(open(os.path.join(CSRC, "mwu_adapters.cu")).read())
    body = text[text.index("mwu_adapters_tile_kernel("):]
    write = body.index("*at = y;")
    branch = body.index("if (rows_here == 32", write)
    assert re.search(r"fence_proxy_async\(\);\s*__syncwarp\(\);", body[write:branch])
    back = body.index("mbar_arrive(smem_u32(&sm->empty[s]))", branch)
    assert body.rindex("uint4 *>(box", 0, back) > branch                 # the last plain read
    assert re.search(r"__syncwarp\(\);\s*if \(lane == 0\) $", body[branch:back])
    assert body.count("mbar_arrive(smem_u32(&sm->empty[s]))") == 2      # here, and where a stage's MMAs are issued
